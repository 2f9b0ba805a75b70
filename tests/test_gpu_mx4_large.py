"""The 4-bit products on the GPU against 64 bits where tests of smaller sizes do not get: bf16 outputs of every tile, persistent
workgroups, rows of H that end inside a run of scales, n-tiles that begin at k-steps of their own, NaN among the large tiles.

Tolerances as in test_gpu_mx4.py: 8 units of 2^-24 of the sum of magnitudes for each matrix instruction of a sum (sum_error), half a
step for each rounding.
"""
import numpy as np
import pytest
import torch

from paper_2605_17889_amd import binding as B
from mx4_large_sizes import (GATEUP_ENDS, GATEUP_LARGE, GATEUP_OWN_KSTEPS, GATEUP_PERSISTENT, LARGE, NAN, OWN_KSTEPS,
                             PERSISTENT)
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", PERSISTENT)
def test_persistent_workgroups(counts, N, K, dtype):
    check_product(offsets_from(counts), N, K, dtype)


@pytest.mark.parametrize("counts,N,K", OWN_KSTEPS)
def test_tiles_that_begin_at_ksteps_of_their_own(counts, N, K):
    check_product(offsets_from(counts), N, K, torch.float32)


@pytest.mark.parametrize("counts,N,K", NAN)
def test_nan_of_a_row_and_of_a_column_and_no_others(counts, N, K):
    """A block of a row, and a block of a weight row, that is NaN: that row and that column of its group, everything else as without."""
    off, E = offsets_from(counts), len(counts)
    R = int(off[-1])
    g = generator(R, E, N, K)
    q, s, _ = random_rows(g, R, K)
    w = [random_rows(g, N, K)[:2] for _ in range(E)]
    wq, ws = torch.stack([m[0] for m in w]), torch.stack([m[1] for m in w])
    ctx = B.MoeContext(R, 512, 128, E, 1)
    new = lambda: torch.empty((R, N), device="cuda")
    call = lambda out: B.moe_gemm_mx4(ctx, q, s, None if E == 1 else cuda(off), R, E, N, K, wq, ws, out)
    want, got = new(), new()
    print(f"gemm with NaN R={R} E={E} N={N} K={K}", flush=True)
    call(want)
    assert torch.isfinite(want).all()
    row, column, e = R // 2, N - 5, E - 1
    s[K // 256, row, 0] = 255                        # the last run's first block
    ws[e, 0, column, 2] = 255                        # block 1
    call(got)
    bad = torch.zeros((R, N), dtype=torch.bool, device="cuda")
    bad[row] = True
    bad[int(off[e]):int(off[e + 1]), column] = True
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], want[~bad])
    ctx.close()


# ---- experts' FFN ------------------------------------------------------------------------------------

def in_4_bits(h, peak):
    """h [rows, f] in blocks of 32 whose largest element is taken to be peak [rows, f / 32]."""
    _, e = torch.frexp(peak)
    unit = torch.exp2(torch.where(peak == 0, -127, (e.long() - 3).clamp(min=-127)).double())[..., None]
    blocks = h.view(h.shape[0], -1, 32)
    m = (blocks / unit).abs()
    code = torch.zeros_like(m, dtype=torch.long)
    for c, tie in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (m > tie) if c % 2 == 0 else (m >= tie)
    return (torch.sign(blocks) * torch.tensor(M.VALUES, device=h.device)[code] * unit).view(h.shape)


def fill_h(ctx, off, R, d, f, E):
    """The memory in which the path keeps H, full of bf16 -infinity: its second byte is 255, a NaN as the scale of a block that nobody
    writes behind a row's end."""
    bf = lambda v, *s: torch.full(s, v, dtype=torch.bfloat16, device="cuda")
    y = bf(0.0, R, d)
    B.moe_expert_ffn(ctx, bf(1e38, R, d), cuda(off), R, bf(1e38, E, f, d), bf(-1e38, E, f, d), bf(1.0, E, d, f), y)
    assert (y == -float("inf")).all()


def check_experts(counts, f, d, nan_row=None):
    off, E = offsets_from(counts), len(counts)
    R = int(off[-1])
    g = generator(R, E, f, d)
    ctx = B.MoeContext(R, d, f, E, 1)
    fill_h(ctx, off, R, d, f, E)
    q, s, x = random_rows(g, R, d)
    # rows of 2^-8 the size and less: arguments of SiLU of a few units
    lower = 10 if d > 4096 else 8
    blocks = torch.zeros_like(s)
    blocks[s > 0] = lower
    s, x = s - blocks, x * 2.0 ** -lower
    # weights in 4 bits, of one expert at a time in 64
    seeds = [generator(R, E, f, e) for e in range(E)]
    weights = lambda gen: [random_rows(gen, n, m) for n, m in ((f, d), (f, d), (d, f))]
    parts = [[m[:2] for m in weights(gen)] for gen in seeds]
    (w1, s1), (w3, s3), (w2, s2) = [[torch.stack([p[m][n] for p in parts]) for n in range(2)] for m in range(3)]
    y = torch.full((R + 1, d), 9.0, dtype=torch.bfloat16, device="cuda")
    print(f"experts counts={counts} f={f} d={d}", flush=True)
    if nan_row is not None:
        s[0, nan_row, 2] = 255
    first = None
    for _ in range(2):                               # the second call finds H as the first one left it
        y[:R] = 3.0
        B.moe_expert_ffn_mx4(ctx, q, s, cuda(off), R, w1, s1, w3, s3, w2, s2, y[:R])
        assert (y[R] == 9).all()
        if first is not None:
            assert torch.equal(y.nan_to_num(7.0), first.nan_to_num(7.0))
        first = y.clone()
    if nan_row is not None:
        assert torch.isnan(y[nan_row]).all()
        y[nan_row] = 0.0
        x[nan_row] = 0.0
    for e in range(E):
        r = slice(int(off[e]), int(off[e + 1]))
        if counts[e] == 0:
            continue
        v1, v3, v2 = (m[2] for m in weights(generator(R, E, f, e)))
        xe = x[r]
        a, u = xe @ v1.t(), xe @ v3.t()
        ea, eu = (sum_error(d) * (xe.abs() @ v.abs().t()) for v in (v1, v3))
        silu = a * torch.sigmoid(a)
        h = silu * u
        # the derivative of SiLU lies in -0.1 .. 1.1; exponential, reciprocal and products are off by a few units, the exponential's
        # argument by half a unit of itself
        eh = 1.1 * ea * (u.abs() + eu) + silu.abs() * eu + (8 + a.abs()) * U * h.abs()
        peak, ep = (v.view(v.shape[0], -1, 32).amax(-1) for v in (h.abs(), eh))
        hq = in_4_bits(h, peak)
        slack = torch.zeros_like(h)                  # another code where an element lies that near to a tie
        for i in (-1, 1):
            for j in (-1, 1):
                slack = torch.maximum(slack, (in_4_bits(h + i * eh, (peak + j * ep).clamp(min=0)) - hq).abs())
        want, loose = hq @ v2.t(), slack @ v2.abs().t()
        tol = sum_error(f) * ((hq.abs() + slack) @ v2.abs().t()) + loose
        tol = tol + BF16 * (want.abs() + tol)
        bad = (y[r].double() - want).abs() > tol
        assert not bad.any(), (e, torch.argwhere(bad)[:4], y[r][bad][:4], want[bad][:4])
    ctx.close()


@pytest.mark.parametrize("counts,f,d", GATEUP_ENDS + GATEUP_LARGE)
def test_rows_of_h_that_end_inside_a_run(counts, f, d):
    check_experts(counts, f, d)


@pytest.mark.parametrize("counts,f,d", GATEUP_PERSISTENT)
def test_experts_of_persistent_workgroups(counts, f, d):
    check_experts(counts, f, d)


@pytest.mark.parametrize("counts,f,d", GATEUP_OWN_KSTEPS)
def test_experts_whose_tiles_begin_at_ksteps_of_their_own(counts, f, d):
    check_experts(counts, f, d)


@pytest.mark.parametrize("counts,f,d", [GATEUP_ENDS[1], GATEUP_LARGE[0], GATEUP_PERSISTENT[0]])
def test_experts_of_a_row_with_nan(counts, f, d):
    check_experts(counts, f, d, nan_row=sum(counts) // 2)


# ---- persistent workgroups in graphs and on two streams ----------------------------------------------

def persistent_work(seed):
    """An FFN and a product that both draw tiles, with the buffers of one caller."""
    counts, f, d = GATEUP_PERSISTENT[0]
    off, E, R = offsets_from(counts), len(counts), sum(counts)
    N = PERSISTENT[0][1]
    g = generator(seed)
    q, s, _ = random_rows(g, R, d)
    w = [[torch.stack(t) for t in zip(*(random_rows(g, n, m)[:2] for _ in range(E)))] for n, m in ((f, d), (f, d), (d, f), (N, d))]
    ctx, offsets = B.MoeContext(R, d, f, E, 1), cuda(off)
    buffers = lambda: (torch.zeros((R, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((R, N), dtype=torch.bfloat16, device="cuda"))

    def work(out, stream=None):
        B.moe_expert_ffn_mx4(ctx, q, s, offsets, R, *w[0], *w[1], *w[2], out[0], stream=stream)
        B.moe_gemm_mx4(ctx, q, s, offsets, R, E, N, d, *w[3], out[1], stream=stream)

    return ctx, q, buffers, work


def test_persistent_workgroups_in_a_graph():
    """Every replay finds the counters as the one before, or an eager call, left them."""
    ctx, q, buffers, work = persistent_work(11)
    work(buffers())
    torch.cuda.synchronize()
    kept = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(kept)
    g = torch.Generator(device="cuda").manual_seed(12)
    for i in range(4):
        q.copy_(torch.randint(0, 256, q.shape, generator=g, device="cuda", dtype=torch.uint8))
        for t in kept:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = buffers()
        work(eager)
        torch.cuda.synchronize()
        for a, b in zip(kept, eager):
            assert torch.equal(a, b) and a.abs().max() > 0, i
    ctx.close()


def test_persistent_workgroups_of_two_contexts_at_once():
    one, two = persistent_work(13), persistent_work(14)
    want = []
    for ctx, q, buffers, work in (one, two):
        want.append(buffers())
        work(want[-1])
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [one[2](), two[2]()]
    torch.cuda.synchronize()
    for _ in range(4):
        for caller, out, stream in zip((one, two), got, streams):
            caller[3](out, stream=stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one[0].close()
    two[0].close()
