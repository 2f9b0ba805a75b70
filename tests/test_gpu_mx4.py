"""The 4-bit path on the GPU against its definitions in 64 bits (oracle/mx4.py).

Tolerances. Operands are exact; the matrix instruction adds 128 products to an fp32 sum, its terms aligned to the largest of
them: off by less than 8 units of 2^-24 of the sum of magnitudes for each instruction, and the parts of a shared reduction
by one more for each of eight. Outputs are rounded once: half a step, torch.finfo(t).eps / 2 of the value.
"""
import numpy as np
import pytest
import torch

from oracle import mx4 as M
from paper_2605_17889_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.finfo(torch.bfloat16).eps / 2
U = 2.0 ** -24


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rows_of(rng, R, K, spread=3, random=False):
    """Rows in 4 bits with blocks of different magnitudes: (codes, scales by block, numbers); random: codes at random."""
    if random:
        q, s = rng.integers(0, 256, (R, K // 2), np.uint8), rng.integers(125, 128, (R, K // 32), np.uint8)
        return q, s, M.decode(q, s)
    x = rng.standard_normal((R, K)) * np.exp2(rng.integers(-spread, spread + 1, (R, K // 32))).repeat(32, 1)
    q, s = M.quantize(x)
    return q, s, M.decode(q, s)


def matrices_of(rng, E, N, K, random=False):
    parts = [rows_of(rng, N, K, random=random) for _ in range(E)]
    return (cuda(np.stack([p[0] for p in parts])), cuda(np.stack([M.arrange(p[1]) for p in parts])),
            np.stack([p[2] for p in parts]))


def sum_error(K):
    return (8 * -(-K // 128) + 8) * U


def offsets_of(rng, R, E, empty=True):
    """Uneven groups, some of them empty."""
    p = rng.random(E) ** 2
    if empty and E > 2:
        p[rng.integers(E)] = 0
    counts = rng.multinomial(R, p / p.sum())
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


# ---- rows -----------------------------------------------------------------------------------------

def special_rows(T, d, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=g).float())
    x = x.to(torch.bfloat16)
    flat = x.view(-1)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.96875, 4.0, -2.5, -0.25, -0.0])
    n = min(flat.numel() // 2, 64)
    flat[:n] = ties.repeat(5)[:n].to(torch.bfloat16)          # ties of a block whose largest element is 7.97
    if T > 3:
        x[1] = 0
        x[2, :32] = float("nan") if d > 32 else 1.0
        x[2, -32:] = torch.finfo(torch.bfloat16).max
        x[3, -1] = float("-inf")
        x[3, 0] = 2.0 ** -133                                 # smallest bf16
    if T > 4:
        x[4] = torch.randint(-3, 4, (d,), generator=g).to(torch.bfloat16) * 2.0 ** -132
    return x


@pytest.mark.parametrize("T,d,gap", [(1, 32, 0), (1, 4096, 0), (7, 64, 1), (9, 224, 3), (5, 256, 0), (17, 288, 5), (33, 1120, 37),
                                     (8, 1408, 0), (64, 6144, 0), (3, 16384, 11), (1025, 512, 8)])
def test_rows_to_4_bits_and_back(T, d, gap):
    wide = torch.full((T, d + gap), 3e38, dtype=torch.bfloat16)
    wide[:, :d] = special_rows(T, d, T * d)
    x = wide.cuda()[:, :d]
    q = torch.full((T, d // 2), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((M.runs(d), T, 8), 0xCD, dtype=torch.uint8, device="cuda")
    y = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    B.moe_quantize_mx4(x, q, s)
    B.moe_dequantize_mx4(q, s, y)
    want_q, want_s = M.quantize(wide[:, :d].double().numpy())
    assert np.array_equal(s.cpu().numpy(), M.arrange(want_s))              # bytes behind the last block too
    assert np.array_equal(q.cpu().numpy(), want_q)
    want = torch.from_numpy(M.decode(want_q, want_s)).to(torch.bfloat16)
    assert torch.equal(y.cpu().view(torch.int16)[~torch.isnan(want)], want.view(torch.int16)[~torch.isnan(want)])
    assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want))


def test_every_code_and_scale_comes_back():
    """All 16 codes under all 256 scales."""
    q = np.tile(np.array([(2 * i) | (2 * i + 1) << 4 for i in range(8)] * 2, np.uint8), (256, 1))
    s = np.arange(256, dtype=np.uint8)[:, None]
    y = torch.empty((256, 32), dtype=torch.bfloat16, device="cuda")
    B.moe_dequantize_mx4(cuda(q), cuda(M.arrange(s)), y)
    want = torch.from_numpy(M.decode(q, s)).to(torch.bfloat16)
    assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want))
    got = y.cpu()
    assert torch.equal(got.view(torch.int16)[:255], want.view(torch.int16)[:255])


# ---- product --------------------------------------------------------------------------------------

def check_product(R, N, K, E=1, fp32=False, seed=0, ctx_rows=None):
    rng = np.random.default_rng(seed + R * 7 + N * 3 + K)
    q, s, x = rows_of(rng, R, K)
    w, ws, wv = matrices_of(rng, E, N, K)
    off = np.array([0, R], np.int32) if E == 1 else offsets_of(rng, R, E)
    ctx = B.MoeContext(ctx_rows or max(R, 1), 512, 128, E, 1)
    out = torch.full((R + 1, N), 77.0, dtype=torch.float32 if fp32 else torch.bfloat16, device="cuda")
    print(f"gemm R={R} N={N} K={K} E={E} fp32={fp32}", flush=True)
    B.moe_gemm_mx4(ctx, cuda(q), cuda(M.arrange(s)), None if E == 1 else cuda(off), R, E, N, K, w, ws, out[:R])
    got = out.double().cpu().numpy()
    assert (got[R] == 77).all()
    for e in range(E):
        r = slice(off[e], off[e + 1])
        want, size = x[r] @ wv[e].T, np.abs(x[r]) @ np.abs(wv[e]).T
        tol = sum_error(K) * size + (U if fp32 else BF16) * np.abs(want) * (1 + 1e-6)
        bad = np.abs(got[r] - want) > tol
        assert not bad.any(), (e, np.argwhere(bad)[:4], got[r][bad][:4], want[bad][:4])
    ctx.close()


@pytest.mark.parametrize("R", [1, 2, 15, 16, 17, 31, 33, 63, 65, 127, 129, 200, 257, 300, 513])
@pytest.mark.parametrize("N,K", [(256, 512), (144, 1408)])
def test_product_rows(R, N, K):
    check_product(R, N, K)


@pytest.mark.parametrize("N", [16, 32, 48, 112, 240, 256, 272, 512, 1040])
@pytest.mark.parametrize("R", [3, 40, 100, 300])
def test_product_columns(R, N):
    check_product(R, N, 768, fp32=True)


@pytest.mark.parametrize("K", [32, 64, 96, 128, 160, 256, 288, 512, 736, 1024, 1312, 2048, 4096, 4128])
@pytest.mark.parametrize("R", [5, 50, 130, 260])
def test_product_reductions(R, K):
    check_product(R, 128, K, fp32=True)


@pytest.mark.parametrize("R,E,N,K", [(1, 4, 64, 512), (13, 5, 96, 544), (64, 8, 128, 1024), (300, 8, 256, 768), (700, 3, 272, 1408),
                                     (1500, 7, 256, 512), (1000, 128, 64, 256), (40, 256, 48, 320)])
def test_product_groups(R, E, N, K):
    check_product(R, N, K, E)


def test_product_of_rows_with_nan_and_no_others():
    rng = np.random.default_rng(5)
    for R in (4, 40, 140, 260):
        q, s, x = rows_of(rng, R, 512)
        s[R // 2, 3] = 255
        w, ws, wv = matrices_of(rng, 1, 64, 512)
        ctx = B.MoeContext(R, 512, 128, 1, 1)
        out = torch.empty((R, 64), dtype=torch.float32, device="cuda")
        B.moe_gemm_mx4(ctx, cuda(q), cuda(M.arrange(s)), None, R, 1, 64, 512, w, ws, out)
        bad = torch.isnan(out).all(1).cpu().numpy()
        assert bad[R // 2] and bad.sum() == 1 and torch.isnan(out).any(1).sum() == 1
        ctx.close()


def test_product_leaves_rows_behind_the_last_group():
    """Groups that hold fewer rows than R."""
    rng = np.random.default_rng(6)
    R, N, K = 90, 64, 256
    q, s, x = rows_of(rng, R, K)
    w, ws, wv = matrices_of(rng, 2, N, K)
    for last in (3, 40, 80):
        off = np.array([0, last // 2, last], np.int32)
        ctx = B.MoeContext(R, 512, 128, 2, 1)
        out = torch.full((R, N), 5.0, dtype=torch.bfloat16, device="cuda")
        B.moe_gemm_mx4(ctx, cuda(q), cuda(M.arrange(s)), cuda(off), R, 2, N, K, w, ws, out)
        assert (out[last:] == 5).all() and not (out[:last] == 5).all()
        ctx.close()


def test_product_of_one_matrix_without_its_axis():
    rng = np.random.default_rng(8)
    q, s, x = rows_of(rng, 9, 256)
    w, ws, wv = matrices_of(rng, 1, 32, 256)
    ctx = B.MoeContext(9, 512, 128, 1, 1)
    a, b = (torch.empty((9, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.moe_gemm_mx4(ctx, cuda(q), cuda(M.arrange(s)), None, 9, 1, 32, 256, w, ws, a)
    B.moe_gemm_mx4(ctx, cuda(q), cuda(M.arrange(s)), None, 9, 1, 32, 256, w[0], ws[0], b)
    assert torch.equal(a, b)
    ctx.close()


# ---- expert FFN -----------------------------------------------------------------------------------

def in_4_bits(h, peak):
    """h [rows, f] in blocks whose largest element is taken to be peak [rows, f / 32]."""
    unit = np.ldexp(1.0, M.scale_bytes(peak).astype(np.int64) - 127)[..., None]
    blocks = h.reshape(h.shape[0], -1, 32)
    return (np.sign(blocks) * M.VALUES[M.codes_of(blocks / unit)] * unit).reshape(h.shape)


def check_experts(T, d, f, E, k, seed=0, off=None, random=False):
    rng = np.random.default_rng(seed + T + d + f + E)
    R = T * k
    q, s, x = rows_of(rng, R, d, 1, random)
    w1, s1, v1 = matrices_of(rng, E, f, d, random)
    w3, s3, v3 = matrices_of(rng, E, f, d, random)
    w2, s2, v2 = matrices_of(rng, E, d, f, random)
    off = offsets_of(rng, R, E) if off is None else off
    ctx = B.MoeContext(T, d, f, E, k)
    y = torch.empty((R, d), dtype=torch.bfloat16, device="cuda")
    print(f"experts T={T} d={d} f={f} E={E} k={k}", flush=True)
    B.moe_expert_ffn_mx4(ctx, cuda(q), cuda(M.arrange(s)), cuda(off), R, w1, s1, w3, s3, w2, s2, y)
    got = y.double().cpu().numpy()
    near_a_tie = 0
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if r.start == r.stop:
            continue
        g, u = x[r] @ v1[e].T, x[r] @ v3[e].T
        eg, eu = (sum_error(d) * (np.abs(x[r]) @ np.abs(v[e]).T) for v in (v1, v3))
        h = M.silu(g) * u
        # the derivative of SiLU lies in -0.1 .. 1.1; exponential, reciprocal and products are off by a few units, the exponential's
        # argument by half a unit of itself
        eh = 1.1 * eg * (np.abs(u) + eu) + np.abs(M.silu(g)) * eu + (8 + np.abs(g)) * U * np.abs(h)
        peak, ep = (v.reshape(v.shape[0], -1, 32).max(-1) for v in (np.abs(h), eh))
        near = np.stack([in_4_bits(h + a * eh, np.maximum(peak + b * ep, 0)) for a in (-1, 1) for b in (-1, 1)])
        hq = in_4_bits(h, peak)
        slack = np.abs(near - hq).max(0)                       # another code where an element lies that near to a tie
        want = hq @ v2[e].T
        tol = sum_error(f) * ((np.abs(hq) + slack) @ np.abs(v2[e]).T) + slack @ np.abs(v2[e]).T
        tol = tol + BF16 * (np.abs(want) + tol)
        bad = np.abs(got[r] - want) > tol
        assert not bad.any(), (e, np.argwhere(bad)[:4], got[r][bad][:4], want[bad][:4])
        near_a_tie += int((slack > 0).sum())
    ctx.close()


@pytest.mark.parametrize("T,d,f,E,k", [(1, 512, 128, 4, 2), (3, 512, 384, 3, 1), (16, 512, 256, 8, 2), (1, 2048, 768, 16, 8),
                                       (40, 1024, 640, 4, 2), (100, 512, 1408, 2, 2), (200, 512, 256, 2, 1), (300, 1024, 384, 3, 2),
                                       (700, 512, 640, 2, 1), (33, 512, 128, 1, 1), (600, 512, 896, 1, 1)])
def test_experts(T, d, f, E, k):
    check_experts(T, d, f, E, k)


def test_experts_of_one_group_only():
    check_experts(70, 512, 256, 4, 1, off=np.array([0, 0, 70, 70, 70], np.int32))


# ---- together, as a layer ---------------------------------------------------------------------------

def layer(T, d, f, E, k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T + d + f + E)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    L = {"x": r(T, d).to(torch.bfloat16), "w_router": r(d, E) * 0.05, "bias": r(E) * 0.1, "correction": r(E) * 0.1}
    for name, n, m in (("w1", f, d), ("w3", f, d), ("w2", d, f)):
        w = (r(E, n, m) * 0.02 * (4 if name != "w2" else 1)).to(torch.bfloat16)
        q = torch.empty((E, n, m // 2), dtype=torch.uint8, device="cuda")
        s = torch.empty((E, M.runs(m), n, 8), dtype=torch.uint8, device="cuda")
        for e in range(E):
            B.moe_quantize_mx4(w[e], q[e], s[e])
        L[name] = [q, s]
    return L


def stages(ctx, L, T, scoring):
    """The layer from the calls that it is made of."""
    d, E, k = ctx.d_model, ctx.E, ctx.k
    R = T * k
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    idx, w, counts, offsets, perm, inv = i32(T, k), torch.empty((T, k), device="cuda"), i32(E), i32(E + 1), i32(R), i32(R)
    if scoring is None:
        B.moe_route(ctx, L["x"], L["w_router"], L["bias"], T, idx, w)
    else:
        B.moe_route_scored(ctx, L["x"], L["w_router"], L["bias"], L["correction"], scoring, T, idx, w)
    xp = torch.empty((R, d), dtype=torch.bfloat16, device="cuda")
    B.moe_permute(ctx, idx, T, counts, offsets, perm, inv, L["x"], xp)
    q, s = u8(R, d // 2), u8(M.runs(d), R, 8)
    B.moe_quantize_mx4(xp, q, s)
    yp, y = torch.empty_like(xp), torch.empty_like(L["x"])
    B.moe_expert_ffn_mx4(ctx, q, s, offsets, R, *L["w1"], *L["w3"], *L["w2"], yp)
    B.moe_combine(ctx, yp, inv, w, T, y)
    return y, idx, w


def whole(ctx, L, T, scoring, y, **kw):
    B.moe_layer_forward_mx4(ctx, L["x"], L["w_router"], L["bias"], None if scoring is None else L["correction"], scoring,
                            *L["w1"], *L["w3"], *L["w2"], T, y, **kw)


@pytest.mark.parametrize("T,d,f,E,k", [(1, 512, 128, 8, 2), (5, 1024, 640, 32, 6), (64, 512, 384, 8, 2), (300, 512, 256, 64, 8),
                                       (1500, 1024, 384, 4, 2)])
@pytest.mark.parametrize("score", [None, "sigmoid", "softmax"])
def test_layer_is_its_stages(T, d, f, E, k, score):
    L = layer(T, d, f, E, k)
    scoring = None if score is None else B.MoeScoring(score, groups=4, top_groups=3 if E > 4 else 2, scale=1.5)
    ctx = B.MoeContext(T, d, f, E, k)
    want, want_idx, want_w = stages(ctx, L, T, scoring)
    y = torch.empty_like(want)
    whole(ctx, L, T, scoring, y)
    assert torch.equal(y, want) and torch.isfinite(y).all() and y.abs().max() > 0
    idx, w = torch.empty_like(want_idx), torch.empty_like(want_w)
    B.moe_last_routing(ctx, T, topk_idx=idx, topk_w=w)
    assert torch.equal(idx, want_idx) and torch.equal(w, want_w)
    # expert outputs kept in fp32: one rounding to bf16 of each of the k less
    B.moe_set_expert_output_fp32(ctx, True)
    z = torch.empty_like(want)
    whole(ctx, L, T, scoring, z)
    size = w.abs().sum(1, keepdim=True) * 8 * y.float().abs().max()
    assert ((z.float() - y.float()).abs() <= BF16 * (size + z.float().abs() + y.float().abs())).all()
    ctx.close()


def test_layer_with_stage_times():
    T, d, f, E, k = 40, 512, 256, 32, 4
    L, scoring = layer(T, d, f, E, k), B.MoeScoring("sigmoid")
    ctx = B.MoeContext(T, d, f, E, k)
    y, z = torch.empty_like(L["x"]), torch.empty_like(L["x"])
    whole(ctx, L, T, scoring, y)
    B.moe_profile_begin(ctx, 2)
    whole(ctx, L, T, scoring, z)
    whole(ctx, L, T, None, z)
    ms, launches, n = B.moe_profile_end(ctx)
    assert n == 2 and all(v > 0 for v in ms.values()) and launches["gateup"] == 2 and launches["gather"] == 2
    whole(ctx, L, T, scoring, z)
    assert torch.equal(y, z)
    ctx.close()


def test_contexts_serve_all_paths_in_turn():
    """The 4-bit path lies in the memory of the bf16 path's intermediates: neither finds the other's there."""
    T, d, f, E, k = 70, 512, 384, 8, 2
    L, scoring = layer(T, d, f, E, k), B.MoeScoring("softmax")
    g = torch.Generator(device="cuda").manual_seed(3)
    W = [(torch.randn(s, generator=g, device="cuda") * 0.05).to(torch.bfloat16) for s in ((E, f, d), (E, f, d), (E, d, f))]
    ctx, alone = B.MoeContext(T, d, f, E, k), B.MoeContext(T, d, f, E, k)
    y4, y16, z4, z16 = (torch.empty_like(L["x"]) for _ in range(4))
    whole(ctx, L, T, scoring, y4)
    B.moe_layer_forward(alone, L["x"], L["w_router"], None, *W, T, y16)
    for _ in range(3):
        B.moe_layer_forward(ctx, L["x"], L["w_router"], None, *W, T, z16)
        whole(ctx, L, T, scoring, z4)
        assert torch.equal(y4, z4) and torch.equal(y16, z16)
    small = L["x"][:9].clone()
    L9 = dict(L, x=small)
    want = stages(alone, L9, 9, scoring)[0]
    z = torch.empty_like(small)
    whole(ctx, L9, 9, scoring, z)
    assert torch.equal(z, want)
    ctx.close()
    alone.close()


@pytest.mark.parametrize("T,E", [(1, 32), (24, 8), (600, 4)])
def test_graph_replays(T, E):
    """Layer, product, rows and router in one graph: every replay gives the eager results of its inputs, with eager work between."""
    d, f, k = 512, 256, 2
    L, scoring = layer(T, d, f, E, k), B.MoeScoring("sigmoid", groups=2, top_groups=1)
    ctx = B.MoeContext(T, d, f, E, k)
    rng = np.random.default_rng(T)
    w, ws, _ = matrices_of(rng, 1, 80, d)
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")

    def buffers():
        return {"y": torch.empty_like(L["x"]), "q": u8(T, d // 2), "s": u8(M.runs(d), T, 8),
                "logits": torch.empty((T, 80), device="cuda"), "back": torch.empty_like(L["x"])}

    def work(b):
        whole(ctx, L, T, scoring, b["y"])
        B.moe_quantize_mx4(b["y"], b["q"], b["s"])
        B.moe_gemm_mx4(ctx, b["q"], b["s"], None, T, 1, 80, d, w, ws, b["logits"])
        B.moe_dequantize_mx4(b["q"], b["s"], b["back"])

    work(buffers())
    torch.cuda.synchronize()
    kept = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(kept)
    g = torch.Generator(device="cuda").manual_seed(T)
    for _ in range(4):
        L["x"].copy_(torch.randn(L["x"].shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = buffers()
        work(eager)
        torch.cuda.synchronize()
        for name in kept:
            assert torch.equal(kept[name], eager[name]), name
    ctx.close()


def test_another_stream_and_two_contexts_at_once():
    T, d, f, E, k = 200, 512, 384, 8, 2
    L, scoring = layer(T, d, f, E, k), B.MoeScoring("sigmoid")
    a, b = B.MoeContext(T, d, f, E, k), B.MoeContext(T, d, f, E, k)
    want = torch.empty_like(L["x"])
    whole(a, L, T, scoring, want)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    y1, y2 = torch.zeros_like(want), torch.zeros_like(want)
    torch.cuda.synchronize()
    for _ in range(5):
        whole(a, L, T, scoring, y1, stream=s1)
        whole(b, L, T, scoring, y2, stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(y1, want) and torch.equal(y2, want)
    a.close()
    b.close()


# ---- refusals that need a context -------------------------------------------------------------------

def test_offsets_past_32_bits():
    """540000 rows of 16384: more than 2^32 bytes of codes and 2^33 elements."""
    T, d, N, last = 540000, 16384, 64, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((last, d), generator=g, device="cuda").to(torch.bfloat16)
    x[-last:] = tail
    q = torch.empty((T, d // 2), dtype=torch.uint8, device="cuda")
    s = torch.empty((M.runs(d), T, 8), dtype=torch.uint8, device="cuda")
    B.moe_quantize_mx4(x, q, s)
    want_q, want_s = torch.empty_like(q[-last:]), torch.empty((M.runs(d), last, 8), dtype=torch.uint8, device="cuda")
    B.moe_quantize_mx4(tail, want_q, want_s)
    assert torch.equal(q[-last:], want_q) and torch.equal(s[:, -last:], want_s)
    B.moe_dequantize_mx4(q, s, x)
    y = torch.empty_like(tail)
    B.moe_dequantize_mx4(want_q, want_s, y)
    assert torch.equal(x[-last:], y) and not x[:-last].any()
    del x
    w, ws, wv = random_rows(g, N, d)
    ctx = B.MoeContext(T, 512, 128, 2, 1)
    out = torch.full((T, N), 5.0, device="cuda")
    want = y.double() @ wv.t()
    tol = sum_error(d) * (y.double().abs() @ wv.abs().t()) + U * want.abs() * (1 + 1e-6)
    for off in (None, [0, T - last, T]):
        E = 1 if off is None else 2
        out.fill_(5.0)
        B.moe_gemm_mx4(ctx, q, s, None if off is None else cuda(np.array(off, np.int32)), T, E, N, d, w.expand(E, -1, -1).contiguous(),
                       ws.expand(E, -1, -1, -1).contiguous(), out)
        assert ((out[-last:].double() - want).abs() <= tol).all() and not out[:-last].any()
    ctx.close()


def test_weights_past_32_bits():
    """Three experts of 2^18 columns: the last one's weights lie behind 2^32 bytes."""
    E, N, K, R = 3, 1 << 18, 16384, 50
    g = torch.Generator(device="cuda").manual_seed(2)
    q, s, x = random_rows(g, R, K)
    w = torch.randint(0, 256, (E, N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    ws = torch.full((E, M.runs(K), N, 8), 127, dtype=torch.uint8, device="cuda")
    ctx = B.MoeContext(R, 512, 128, E, 1)
    out = torch.empty((R, N), device="cuda")
    values = torch.tensor(np.concatenate([M.VALUES, -M.VALUES]), device="cuda")
    for rows in (R, 3):                              # of the last expert
        B.moe_gemm_mx4(ctx, q, s, cuda(np.array([0, 0, R - rows, R], np.int32)), R, E, N, K, w, ws, out)
        for e, r in ((1, slice(0, R - rows)), (2, slice(R - rows, R))):
            cols = slice(N - 40, N)
            wv = values[torch.stack((w[e, cols] & 15, w[e, cols] >> 4), dim=-1).long()].flatten(-2)
            want = x[r] @ wv.t()
            tol = sum_error(K) * (x[r].abs() @ wv.abs().t()) + U * want.abs() * (1 + 1e-6)
            assert ((out[r, cols].double() - want).abs() <= tol).all()
    ctx.close()


def test_a_row_for_each_of_256_groups_and_the_most_columns():
    """Small tiles would be more than a launch holds: 272 row tiles through 2^22 columns."""
    E, N, K = 256, 1 << 22, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    q, s, x = random_rows(g, E, K)
    w = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    for e in range(E):
        w[e] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    ws = torch.zeros((E, 1, N, 8), dtype=torch.uint8, device="cuda")
    ws[..., 0] = 127
    out = torch.full((E, N), 77.0, dtype=torch.bfloat16, device="cuda")
    ctx = B.MoeContext(E, 512, 128, E, 1)
    B.moe_gemm_mx4(ctx, q, s, torch.arange(E + 1, dtype=torch.int32, device="cuda"), E, E, N, K, w, ws, out)
    values = torch.tensor(np.concatenate([M.VALUES, -M.VALUES]), device="cuda")
    for cols in (slice(0, 100), slice(N // 2 - 50, N // 2 + 50), slice(N - 100, N)):
        wv = values[torch.stack((w[:, cols] & 15, w[:, cols] >> 4), dim=-1).long()].flatten(-2)
        want = (x[:, None] * wv).sum(-1)
        tol = sum_error(K) * (x[:, None].abs() * wv.abs()).sum(-1) + BF16 * want.abs() * (1 + 1e-6)
        assert ((out[:, cols].double() - want).abs() <= tol).all()
    ctx.close()


def test_refusals():
    ctx = B.MoeContext(8, 512, 128, 4, 2)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(5, dtype=torch.int32, device="cuda")

    def gemm(R=4, E=1, N=64, K=256, offsets=None, shift=0, out=None):
        take = lambda *s: u8(int(np.prod(s)) + 16)[shift:shift + int(np.prod(s))].view(*s)
        B.moe_gemm_mx4(ctx, take(R, K // 2), u8(M.runs(K), R, 8), offsets, R, E, N, K, u8(E, N, K // 2), u8(E, M.runs(K), N, 8),
                       bf(R, N) if out is None else out)

    gemm()
    gemm(R=0)
    with pytest.raises(B.MoeError, match="INVALID_ARG"):
        gemm(R=17)                                   # more rows than T_max * k
    with pytest.raises(B.MoeError, match="INVALID_ARG"):
        gemm(E=4)                                    # groups without offsets
    with pytest.raises(B.MoeError, match="INVALID_ARG"):
        gemm(shift=8)                                # rows that do not start at 16 bytes
    with pytest.raises(B.MoeError, match="INVALID_ARG"):
        gemm(out=bf(4 * 64 + 8)[4:4 + 256].view(4, 64))
    for change in (dict(N=24), dict(N=8), dict(K=48), dict(K=16)):
        with pytest.raises(B.MoeError, match="UNSUPPORTED_SHAPE"):
            gemm(**change)
    with pytest.raises(B.MoeError):
        gemm(out=torch.zeros((4, 64), dtype=torch.float16, device="cuda"))
    logits, idx, w = torch.zeros((4, 4), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    for kw in (dict(groups=3), dict(groups=0), dict(groups=4, top_groups=1), dict(groups=2, top_groups=3), dict(groups=2, top_groups=0),
               dict(group_best=0), dict(group_best=3), dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(B.MoeError, match="INVALID_ARG"):
            B.moe_route_scored_from_logits(ctx, logits, None, B.MoeScoring("sigmoid", **kw), 4, idx, w)
    with pytest.raises(B.MoeError, match="INVALID_ARG"):
        B.moe_route_scored_from_logits(ctx, logits, None, None, 4, idx, w)
    L = layer(4, 512, 128, 4, 2)
    with pytest.raises(B.MoeError, match="INVALID_ARG"):           # a correction without scores that it could correct
        B.moe_layer_forward_mx4(ctx, L["x"], L["w_router"], None, L["correction"], None, *L["w1"], *L["w3"], *L["w2"], 4, bf(4, 512))
    ctx.close()
    many = B.MoeContext(4, 512, 128, 256, 2)
    with pytest.raises(B.MoeError, match="UNSUPPORTED_SHAPE"):
        B.moe_route_scored_from_logits(many, torch.zeros((4, 256), device="cuda"), None, B.MoeScoring("sigmoid", groups=128, top_groups=4),
                                       4, idx, w)
    many.close()


# ---- every tile, at sizes too large for the host -----------------------------------------------------

from mx4_sizes import GATEUP, PLAIN  # noqa: E402


def random_rows(g, *lead):
    """Codes at random and scales of five magnitudes, on the GPU: (codes, arranged scales, numbers in 64 bits)."""
    *front, rows, K = lead
    q = torch.randint(0, 256, (*front, rows, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    blocks = K // 32
    s = torch.randint(125, 130, (*front, rows, blocks), generator=g, device="cuda", dtype=torch.uint8)
    whole = torch.zeros((*front, rows, M.runs(K) * 8), dtype=torch.uint8, device="cuda")
    whole[..., :blocks] = s
    arranged = whole.view(*front, rows, -1, 2, 4).transpose(-1, -2).movedim(-4, -3).reshape(*front, -1, rows, 8).contiguous()
    values = torch.tensor(np.concatenate([M.VALUES, -M.VALUES]), device="cuda")
    v = values[torch.stack((q & 15, q >> 4), dim=-1).long()].flatten(-2)
    return q, arranged, (v.view(*front, rows, blocks, 32) * torch.exp2(s.double() - 127)[..., None]).flatten(-2)


@pytest.mark.parametrize("R,E,N,K", PLAIN)
def test_product_of_every_tile(R, E, N, K):
    g = torch.Generator(device="cuda").manual_seed(R + E + N + K)
    rng = np.random.default_rng(R + E + N + K)
    q, s, x = random_rows(g, R, K)
    off = np.array([0, R], np.int32) if E == 1 else offsets_of(rng, R, E)
    w = [random_rows(g, N, K) for _ in range(E)]
    ctx = B.MoeContext(R, 512, 128, E, 1)
    out = torch.full((R + 2, N), 9.0, device="cuda")
    print(f"gemm R={R} E={E} N={N} K={K}", flush=True)
    for _ in range(2):                               # the second call finds counters as the first one left them
        out[:R] = 3.0
        B.moe_gemm_mx4(ctx, q, s, None if E == 1 else cuda(off), R, E, N, K, torch.stack([m[0] for m in w]),
                       torch.stack([m[1] for m in w]), out[:R])
        assert (out[R:] == 9).all()
        for e in range(E):
            r = slice(int(off[e]), int(off[e + 1]))
            want = x[r] @ w[e][2].t()
            tol = sum_error(K) * (x[r].abs() @ w[e][2].abs().t()) + U * want.abs() * (1 + 1e-6)
            assert ((out[r].double() - want).abs() <= tol).all(), (e, (out[r].double() - want).abs().max())
    ctx.close()


@pytest.mark.parametrize("R,E,f,d", GATEUP)
def test_experts_of_every_tile(R, E, f, d):
    check_experts(R, d, f, E, 1, seed=1, random=True)
