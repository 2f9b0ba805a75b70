"""Rows in 8 bits: moe_rmsnorm_i8 and moe_quantize_i8 against the definition in 64 bits.

Tolerances, counted in roundings (half a step: 2^-24 in fp32, 2^-8 in bf16, relative to the value):
  h          one fp32 addition, then the rounding to residual_out's type
  statistic  the sum of d squares is a chain of at most 8 * CHUNKS = 64 fused multiply-adds in a thread, 6 additions in a
             wavefront and 16 over wavefronts: 86 roundings, halved by the root; with the division, the root, the
             reciprocal, h's own rounding and the two products 43 + 8 -> ROOT = 51 roundings of 2^-24
  y, scale   the statistic, then the output's own rounding
  q          |q - v / scale| <= 1/2, of values up to 127 that are off by ROOT + 3 roundings of 2^-24
"""
import pytest
import torch

from paper_2605_17889_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-6
HALF32, HALF16 = 2.0 ** -24, 2.0 ** -8
ROOT = 51 * HALF32
TINY = 2.0 ** -126           # below the normal range the step is absolute


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(T, d, residual, gap=0, seed=0, scale=1.0):
    g = gen(seed)
    wide = (torch.randn((T, d + gap), generator=g, device="cuda") * scale).to(torch.bfloat16)
    x = wide[:, gap // 2:gap // 2 + d]
    res = None
    if residual is not None:
        res = (torch.randn((T, d), generator=g, device="cuda") * 3 * scale).to(residual)
    w = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
    return x, res, w


def outputs(T, d, residual):
    h = torch.empty((T, d), dtype=residual, device="cuda") if residual is not None else None
    return (h, torch.empty((T, d), dtype=torch.bfloat16, device="cuda"),
            torch.full((T, d), 77, dtype=torch.int8, device="cuda"), torch.full((T,), -1.0, device="cuda"))


def exact(x, res, w, eps=EPS):
    h = x.double() if res is None else x.double() + res.double()
    return h, h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w.double()


def near(got, want, rel, tiny=TINY):
    off = (got.double() - want).abs() - (want.abs() * rel + tiny)
    assert off.numel() == 0 or off.max().item() <= 0, f"off by {off.max().item():.3g} more than allowed"


def check_q(q, scale, v, rel):
    peak = v.abs().amax(1)
    near(scale, peak / 127, rel)
    t = torch.where(peak[:, None] > 0, v * 127 / peak[:, None].clamp(min=1e-300), 0.0)
    assert (q.double() - t).abs().max().item() <= 0.5 + 127 * (ROOT + 3 * HALF32)
    assert q.min().item() >= -127


def check(x, res, w, got, eps=EPS):
    h, v = exact(x, res, w, eps)
    res_out, y, q, scale = got
    if res_out is not None:
        half = HALF32 if res_out.dtype == torch.float32 else HALF16
        near(res_out, h, (half + HALF32) * (1 + HALF16))
    if y is not None:
        near(y, v, (HALF16 + ROOT) * (1 + HALF16))
    if q is not None:
        check_q(q, scale, v, ROOT + 2 * HALF32)


KINDS = {"none": None, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 8), (2, 9), (1, 64), (6, 511), (4, 512), (3, 513), (257, 1111),
                                 (1, 2048), (5, 2056), (1, 4096), (7, 6144), (2, 8200), (3, 16384), (2, 16392),
                                 (1, 65535), (2, 65536), (300, 24), (1030, 2048), (2100, 1000)])
def test_norm(T, d, kind):
    x, res, w = make(T, d, KINDS[kind], seed=T * 7 + d)
    got = outputs(T, d, KINDS[kind])
    B.moe_rmsnorm_i8(x, res, w, EPS, *got)
    check(x, res, w, got)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gap", [1, 2, 8, 37])
def test_norm_of_rows_cut_out_of_a_wider_tensor(gap, kind):
    for T, d in ((1, 40), (9, 1111), (33, 2048), (5, 6144)):
        x, res, w = make(T, d, KINDS[kind], gap=gap, seed=gap)
        got = outputs(T, d, KINDS[kind])
        B.moe_rmsnorm_i8(x, res, w, EPS, *got)
        check(x, res, w, got)


@pytest.mark.parametrize("d", [100, 1111, 6144])
def test_norm_in_place_and_with_outputs_left_out(d):
    for kind in ("bf16", "fp32"):
        x, res, w = make(17, d, KINDS[kind], seed=3)
        full = outputs(17, d, KINDS[kind])
        B.moe_rmsnorm_i8(x, res, w, EPS, *full)
        stream = res.clone()
        B.moe_rmsnorm_i8(x, stream, w, EPS, residual_out=stream)
        assert torch.equal(stream, full[0])
        _, y, q, scale = outputs(17, d, None)
        B.moe_rmsnorm_i8(x, res, w, EPS, y=y)
        B.moe_rmsnorm_i8(x, res, w, EPS, q=q, q_scale=scale)
        for a, b in zip((y, q, scale), full[1:]):
            assert torch.equal(a, b)
    # without a residual the sum is x itself, in either type
    x, _, w = make(17, d, None, seed=4)
    for kind in (torch.bfloat16, torch.float32):
        h = torch.empty((17, d), dtype=kind, device="cuda")
        B.moe_rmsnorm_i8(x, None, w, EPS, residual_out=h)
        assert torch.equal(h, x.to(kind))


@pytest.mark.parametrize("d", [8, 1111, 6144, 20000])
def test_norm_of_zero_infinite_and_nan_rows(d):
    x, res, w = make(8, d, torch.float32, seed=5)
    clean = outputs(8, d, torch.float32)
    B.moe_rmsnorm_i8(x, res, w, EPS, *clean)
    x, res = x.clone(), res.clone()
    x[1] = 0
    res[1] = 0
    x[3, d - 1] = float("inf")
    res[4, 0] = float("nan")
    x[6, d // 2], res[6, d // 2] = float("inf"), float("-inf")
    got = outputs(8, d, torch.float32)
    B.moe_rmsnorm_i8(x, res, w, EPS, *got)
    h, y, q, scale = got
    assert scale[1].item() == 0 and not q[1].any() and not y[1].any()
    for bad in (3, 4, 6):
        assert scale[bad].isnan() and not q[bad].any()
        assert not y[bad].isfinite().all()
    for t in (0, 2, 5, 7):
        for a, b in zip(got, clean):
            assert torch.equal(a[t], b[t])


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e18, 1e25, 1e36])
@pytest.mark.parametrize("d", [64, 1111, 8192])
def test_norm_of_very_small_and_very_large_values(d, scale):
    """Squares past the range of fp32 and below it: the result is that of 64 bits."""
    x, res, w = make(5, d, torch.bfloat16, seed=6, scale=scale)
    for eps in (EPS, 1e-30):
        got = outputs(5, d, torch.bfloat16)
        B.moe_rmsnorm_i8(x, res, w, eps, *got)
        _, v = exact(x, res, w, eps)
        if scale == 1e-30 and eps == 1e-30:        # squares of 1e-60 are zero in fp32: eps alone is left, as it is in 64 bits
            assert (v.abs().max() < 1e-13).item()
        check(x, res, w, got, eps)


@pytest.mark.parametrize("T,d", [(1, 1), (4, 9), (3, 768), (300, 1408), (1, 14336), (70, 14336), (2, 65536), (5, 4104)])
@pytest.mark.parametrize("gap", [0, 3])
def test_quantize(T, d, gap):
    x, _, _ = make(T, d, None, gap=gap, seed=d)
    _, _, q, scale = outputs(T, d, None)
    B.moe_quantize_i8(x, q, scale)
    check_q(q, scale, x.double(), 2 * HALF32)


def test_quantize_ties_extremes_and_odd_rows():
    x = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda")
    x[0] = torch.arange(64, device="cuda") + 0.5            # with 127 as the largest: halves go to the even neighbour
    x[0, 63] = 127
    x[1] = torch.arange(64, device="cuda") * 2.0 ** -133    # subnormal bf16
    x[2] = torch.linspace(-3.3e38, 3.3e38, 64, device="cuda").to(torch.bfloat16)
    x[4, 5] = float("nan")
    x[5, 63] = float("-inf")
    x[6] = 1e-37
    _, _, q, scale = outputs(8, 64, None)
    B.moe_quantize_i8(x, q, scale)
    assert torch.equal(q[0].float(), torch.round(x[0].float()))
    assert scale[0].item() == 1
    finite = [t for t in (2, 3, 6, 7) if x[t].isfinite().all()]    # (linspace over this range overflows in fp32)
    check_q(q[finite], scale[finite], x[finite].double(), 2 * HALF32)
    assert scale[2].isfinite() == x[2].isfinite().all()
    # the scale of subnormal rows is itself subnormal: half a step of 2^-149 on 63 * 2^-133 / 127
    assert torch.equal(q[1].double(), torch.round(x[1].double() * 127 / x[1].double().abs().max()))
    near(scale[1:2], x[1:2].double().abs().amax(1) / 127, 2 * HALF32, 2.0 ** -150)
    assert scale[4].isnan() and scale[5].isnan() and not q[4].any() and not q[5].any()
    assert scale[3].item() == 0 and not q[3].any()


def test_quantize_up_to_the_largest_bf16():
    x = (torch.linspace(-1, 1, 256, device="cuda") * 3.38e38).to(torch.bfloat16)[None].repeat(3, 1)
    assert x.isfinite().all()
    _, _, q, scale = outputs(3, 256, None)
    B.moe_quantize_i8(x, q, scale)
    check_q(q, scale, x.double(), 2 * HALF32)


def test_rows_past_32_bit_offsets():
    """2^32 elements and more: the last rows are what a call of them alone gives."""
    T, d = 70000, 65536
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    x.view(-1)[:1 << 16].normal_(generator=gen(7))
    x[:] = x[0]
    x[-3:].normal_(generator=gen(8))
    q, scale = torch.empty((T, d), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    B.moe_quantize_i8(x, q, scale)
    check_q(q[-3:], scale[-3:], x[-3:].double(), 2 * HALF32)
    assert torch.equal(q[T // 2], q[0])
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    B.moe_rmsnorm_i8(x, None, w, EPS, q=q, q_scale=scale)
    check(x[-3:], None, w, (None, None, q[-3:], scale[-3:]))


def test_graph_replays_and_other_streams():
    x, res, w = make(64, 2048, torch.bfloat16, seed=9)
    got = outputs(64, 2048, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.moe_rmsnorm_i8(x, res, w, EPS, *got, stream=side)
    side.synchronize()
    check(x, res, w, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_rmsnorm_i8(x, res, w, EPS, *got)
    for seed in (10, 11, 12):
        a, b, _ = make(64, 2048, torch.bfloat16, seed=seed)
        x.copy_(a)
        res.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        check(x, res, w, got)


def test_no_rows():
    x, res, w = make(0, 64, torch.bfloat16)
    B.moe_rmsnorm_i8(x, res, w, EPS, *outputs(0, 64, torch.bfloat16))
    B.moe_quantize_i8(x, *outputs(0, 64, None)[2:])
    torch.cuda.synchronize()


def test_binding_refuses_other_tensors():
    x, res, w = make(4, 64, torch.bfloat16)
    h, y, q, scale = outputs(4, 64, torch.bfloat16)
    for args in ((x.float(), res, w, EPS, h, y), (x.t(), res, w, EPS, h, y), (x, res[:2], w, EPS, h, y),
                 (x, res, w[:8], EPS, h, y), (x, res, w, EPS, h.float(), y), (x, res, w, EPS, h, y.t()),
                 (x, res, w, EPS, h, y, q.float(), scale), (x, res, w, EPS, h, y, q, scale[:2]),
                 (x, res, w, EPS, h, y, q, None), (x, res, w, 0.0, h, y), (x, res, None, EPS, h, y),
                 (x, res, w, float("nan"), h, y), (x, res, w, EPS), (x, res.half(), w, EPS, None, y),
                 (x[:1].expand(4, 64), res, w, EPS, h, y), (x.cpu(), res, w, EPS, h, y)):
        with pytest.raises(B.MoeError):
            B.moe_rmsnorm_i8(*args)
    for args in ((x.float(), q, scale), (x, q[:2], scale), (x, q, scale[:1]), (x, None, scale), (x, q, None)):
        with pytest.raises(B.MoeError):
            B.moe_quantize_i8(*args)


@pytest.mark.parametrize("d", [1, 8, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 512, 520, 1024, 1032, 1536, 1544, 2048, 2049, 4096, 4104, 6152, 8192, 8193, 16385, 32768, 32769])
def test_every_width_class(d):
    for T in (1, 5, 67):
        x, res, w = make(T, d, torch.bfloat16, gap=3, seed=d)
        got = outputs(T, d, torch.bfloat16)
        B.moe_rmsnorm_i8(x, res, w, EPS, *got)
        check(x, res, w, got)
        _, _, q, scale = outputs(T, d, None)
        B.moe_quantize_i8(x, q, scale)
        check_q(q, scale, x.double(), 2 * HALF32)


def test_more_rows_than_a_launch_has_threads_for():
    """2^20 rows and more of 1024 threads each are several launches: rows on both sides of the border, in every tensor."""
    T, d = (1 << 20) + 5, 8200
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    x[:] = torch.randn(d, generator=gen(1), device="cuda").bfloat16()
    near_border = slice((1 << 20) - 3, T)
    x[near_border] = torch.randn((8, d), generator=gen(2), device="cuda").bfloat16()
    q, scale = torch.empty((T, d), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    B.moe_quantize_i8(x, q, scale)
    for rows in (slice(0, 3), near_border):
        check_q(q[rows], scale[rows], x[rows].double(), 2 * HALF32)
    assert torch.equal(q[1000], q[0]) and torch.equal(scale[:(1 << 20) - 3], scale[:1].expand((1 << 20) - 3))
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    h, y = torch.empty_like(x), torch.empty_like(x)
    B.moe_rmsnorm_i8(x, x, w, EPS, h, y, q, scale)
    for rows in (slice(0, 3), near_border):
        check(x[rows], x[rows], w, (h[rows], y[rows], q[rows], scale[rows]))


@pytest.mark.parametrize("d", [1, 5, 7, 8, 9, 15, 61, 509, 1021, 1111, 2047, 4093, 8191, 16383, 32767, 65521, 65529, 65531, 65535])
def test_odd_widths_at_every_alignment(d):
    """Rows of odd widths, from any element on and in place; nothing beside them is written."""
    T = 17
    for kind in (None, torch.bfloat16, torch.float32):
        x, res, w = make(T, d, kind, gap=5, seed=d)
        flat = [torch.full((T * d + 64,), 7, dtype=t, device="cuda") if t is not None else None
                for t in (kind, torch.bfloat16, torch.int8)]
        for start in (0, 1, 8):
            for f in flat:
                if f is not None:
                    f.fill_(7)
            h, y, q = (None if f is None else f[start + 8:start + 8 + T * d].view(T, d) for f in flat)
            scale = torch.full((T,), -1.0, device="cuda")
            B.moe_rmsnorm_i8(x, res, w, EPS, h, y, q, scale)
            check(x, res, w, (h, y, q, scale))
            if res is not None:
                stream = res.clone()
                B.moe_rmsnorm_i8(x, stream, w, EPS, residual_out=stream, y=(again := torch.empty_like(y)))
                assert torch.equal(stream, h) and torch.equal(again, y)
            for f in flat:
                assert f is None or ((f[:start + 8] == 7).all() and (f[start + 8 + T * d:] == 7).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("largest", [1e37, 3e38])
@pytest.mark.parametrize("d", [64, 1111, 8192, 65536])
def test_norm_of_values_up_to_the_largest(d, largest, kind):
    """Rows whose sum of squares leaves the range of fp32 by up to 2^144: the result is that of 64 bits. Their scaling is by a power
    of two, so the tolerances are the usual ones."""
    T, g = 6, gen(d)
    whole = (torch.rand((T, d), generator=g, device="cuda") * 2 - 1) * largest
    whole[1] = largest                                   # all alike: the largest sum
    whole[2] = torch.randn(d, generator=g, device="cuda")
    whole[2, d - 1] = largest                            # one beside ordinary ones
    whole[3] = torch.randn(d, generator=g, device="cuda")          # no such value at all
    _, _, w = make(1, d, None, seed=d)
    x = (whole if KINDS[kind] is None else whole / 2).bfloat16()
    res = None if KINDS[kind] is None else (whole / 2).to(KINDS[kind])
    got = outputs(T, d, KINDS[kind])
    B.moe_rmsnorm_i8(x, res, w, EPS, *got)
    assert got[2].abs().amax(1).eq(127).all() and (got[3] > 0).all()
    check(x, res, w, got)


def rows_with_ties(rows, d, seed):
    """bf16 rows, the largest element's mantissa every one of the 128 in turn, with its halves and other short fractions of it
    (among which, for bf16 rows, the halves alone are ties unless the mantissa is that of 127)."""
    g = gen(seed)
    peak = (1 + torch.arange(rows, device="cuda") % 128 / 128.0) * 2.0 ** (torch.arange(rows, device="cuda") // 128 % 7 * 30 - 90)
    part = torch.rand((rows, d), generator=g, device="cuda") * 2 - 1
    part[:, ::3] = torch.randint(-256, 257, (rows, (d + 2) // 3), generator=g, device="cuda") / 256.0
    part[:, 1], part[:, d // 2], part[:, d - 1] = 0.5, -0.5, 1.0
    return (part * peak[:, None]).bfloat16()


def test_ties_go_to_even_in_every_row():
    """q is what 64 bits give, bit for bit: a product of 127 and a bf16 number is exact there, and a quotient of such numbers that
    is no tie differs from one by 1 / (2 * 255 * 127) of itself or more, far more than any rounding."""
    for d in (64, 1111, 4096):
        x = rows_with_ties(7 * 128, d, seed=d)
        _, y, q, scale = outputs(7 * 128, d, None)
        want = (x.double() * 127 / x.double().abs().amax(1, keepdim=True)).round()
        assert (want[:, 1] == 64).all() and (want[:, d // 2] == -64).all()
        B.moe_quantize_i8(x, q, scale)
        assert torch.equal(q.double(), want)
        # the norm, weights of one: u is the row itself
        q.fill_(77)
        B.moe_rmsnorm_i8(x, None, torch.ones(d, dtype=torch.bfloat16, device="cuda"), EPS, y=y, q=q, q_scale=scale)
        assert torch.equal(q.double(), want)


def test_norm_that_falls_below_the_range_is_a_row_of_zeros():
    """Values so small beside eps that v is zero in fp32: scale 0 and q 0, as for every row of zeros."""
    x = torch.zeros((4, 200), dtype=torch.bfloat16, device="cuda")
    x[1], x[2, 7], x[3] = 1e-36, -1e-37, 1.0
    w = torch.ones(200, dtype=torch.bfloat16, device="cuda")
    _, y, q, scale = outputs(4, 200, None)
    B.moe_rmsnorm_i8(x, None, w, 1e30, y=y, q=q, q_scale=scale)
    assert not scale[:3].any() and not q[:3].any() and not y[:3].any()
    check(x[3:], None, w, (None, y[3:], q[3:], scale[3:]), 1e30)
