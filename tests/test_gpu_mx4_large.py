"""The 4-bit products on the GPU against 64 bits where tests of smaller sizes do not get: bf16 outputs of every tile, large
tiles of every height.

Tolerances as in test_gpu_mx4.py: 8 units of 2^-24 of the sum of magnitudes for each matrix instruction of a sum (sum_error), half a
step for each rounding.
"""
import numpy as np
import pytest
import torch

from paper_2605_17889_amd import binding as B
from mx4_large_sizes import LARGE
from mx4_sizes import PLAIN
from oracle import mx4 as M
from test_gpu_mx4 import BF16, U, cuda, offsets_of, random_rows, sum_error

pytestmark = pytest.mark.gpu


def offsets_from(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def generator(*seed):
    return torch.Generator(device="cuda").manual_seed(int(np.dot(seed, (1, 3, 7, 31)[:len(seed)])))


# ---- products --------------------------------------------------------------------------------------

def check_product(off, N, K, dtype):
    R, E = int(off[-1]), len(off) - 1
    g = generator(R, E, N, K)
    q, s, x = random_rows(g, R, K)
    w = [random_rows(g, N, K) for _ in range(E)]
    wq, ws = torch.stack([m[0] for m in w]), torch.stack([m[1] for m in w])
    ctx = B.MoeContext(R, 512, 128, E, 1)
    out = torch.full((R + 2, N), 9.0, dtype=dtype, device="cuda")
    step = U if dtype is torch.float32 else BF16
    print(f"gemm R={R} E={E} N={N} K={K} {dtype}", flush=True)
    first = None
    for _ in range(3):                               # later calls find counters as the ones before left them
        out[:R] = 3.0
        B.moe_gemm_mx4(ctx, q, s, None if E == 1 else cuda(off), R, E, N, K, wq, ws, out[:R])
        assert (out[R:] == 9).all()
        if first is None:
            first = out.clone()
            for e in range(E):
                r = slice(int(off[e]), int(off[e + 1]))
                want, size = x[r] @ w[e][2].t(), x[r].abs() @ w[e][2].abs().t()
                tol = sum_error(K) * size
                tol = tol + step * (want.abs() + tol)
                assert ((out[r].double() - want).abs() <= tol).all(), (e, (out[r].double() - want).abs().max())
        else:
            assert torch.equal(out, first)
    ctx.close()


@pytest.mark.parametrize("R,E,N,K", PLAIN)
def test_bf16_outputs_of_every_tile(R, E, N, K):
    off = np.array([0, R], np.int32) if E == 1 else offsets_of(np.random.default_rng(R + E + N + K), R, E)
    check_product(off, N, K, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", LARGE)
def test_large_tiles_of_every_height(counts, N, K, dtype):
    check_product(offsets_from(counts), N, K, dtype)
