"""Operators of the 8-bit path of a Mixture-of-Experts block, as a program that serves such blocks
calls them:

  norm     residual addition, root-mean-square norm and 8-bit rows with a scale each: what stands in
           front of every 8-bit product (moe_rmsnorm_i8)
  gemm     matrix product of 8-bit integers with a scale for each token and each output channel, one
           matrix or one per expert over rows grouped by expert (moe_gemm_i8)
  experts  the gated feed-forward network of all experts over 8-bit rows grouped by expert
           (moe_expert_ffn_i8): two products with SiLU(gate) * up between them, rounded to bf16 and
           brought to 8 bits again row by row, as the operator is defined

Layer shapes are this repository's presets (paper_2605_17889_amd/synth.py) or generic.
"""
import math

import torch

own = False

# d_model, d_ff, experts, experts per token
SHAPES = {
    "tiny": (512, 1024, 8, 2),
    "mixtral8x7b": (4096, 14336, 8, 2),
    "mixtral8x22b": (6144, 16384, 8, 2),
    "qwen3_30b_a3b": (2048, 768, 128, 8),
    "deepseek_v2_lite": (2048, 1408, 64, 6),
}
EPS = 1e-6


def _norm(T, d, residual="bf16", gap=0):
    return {"op": "norm", "T": T, "d": d,
            "residual": residual,          # none | bf16 | fp32: type of the residual stream
            "gap": gap}                    # elements between the rows of x (x is part of a wider tensor)


def _gemm(T, K, N, E=1, out="bf16"):
    return {"op": "gemm", "T": T, "K": K, "N": N, "E": E, "out": out}


def _experts(shape, T, skew=0.0):
    d, f, E, k = SHAPES[shape]
    return {"op": "experts", "shape": shape, "T": T, "d_model": d, "d_ff": f, "E": E, "k": k,
            "skew": skew}                  # expert load ~ rank^-skew


def listed():
    named = lambda name, case: {"name": name, **case}
    return [
        # decode of a single sequence: the norm is all latency
        named("norm_t1_d4096", _norm(1, 4096)),
        # a ragged batch of an odd width, rows cut out of a wider tensor, residual stream in fp32
        named("norm_t1003_d1111_strided", _norm(1003, 1111, residual="fp32", gap=37)),
        # the headline prefill chunk
        named("norm_t8192_d6144", _norm(8192, 6144)),
        # decode of a single sequence through one projection with a long reduction: weights stream by
        named("gemm_t1_k14336_n4096", _gemm(1, 14336, 4096)),
        # a ragged decode batch through a wide matrix, fp32 outputs (logits of a head)
        named("gemm_t37_k2048_n32000_fp32", _gemm(37, 2048, 32000, out="fp32")),
        # a ragged prefill chunk of a few hundred tokens through an attention-sized projection
        named("gemm_t1003_k4096_n6144", _gemm(1003, 4096, 6144)),
        # the headline prefill chunk through one dense projection
        named("gemm_t8192_k6144_n16384", _gemm(8192, 6144, 16384)),
        # the smallest layer the repository knows: launches and latency
        named("experts_tiny_t256", _experts("tiny", 256)),
        # decode of a single sequence: eight of 128 experts hold a row, all other groups are empty
        named("experts_qwen3_t1", _experts("qwen3_30b_a3b", 1)),
        # batched decode through large experts: all weights are read for a handful of rows each
        named("experts_mixtral8x7b_t16", _experts("mixtral8x7b", 16)),
        # prefill of a ragged number of tokens through many small experts, loads as skewed as routers skew them
        named("experts_qwen3_t5003_skewed", _experts("qwen3_30b_a3b", 5003, skew=0.5)),
        # the headline prefill chunk
        named("experts_mixtral8x22b_t8192", _experts("mixtral8x22b", 8192)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gemm", "gemm", "experts", "experts"])
    if op == "norm":
        d = rng.choice([_log_int(rng, 64, 16384), 8 * _log_int(rng, 16, 2048)])
        T = min(_log_int(rng, 1, 16384), (8192 * 6144) // d)
        return _norm(T, d, rng.choice(["none", "bf16", "fp32"]), rng.choice([0, 0, rng.randint(1, 512)]))
    if op == "gemm":
        E = rng.choice([1, 1, 1, rng.randint(2, 32)])
        K = 128 * _log_int(rng, 2, 128)
        N = 128 * _log_int(rng, 1, 256 if E == 1 else 32)
        T = min(_log_int(rng, 1, 8192), int(8192 * 6144 * 16384 / (K * N)))
        return _gemm(T, K, N, E, rng.choice(["bf16", "bf16", "fp32"]))
    shape = rng.choice(sorted(SHAPES))
    return _experts(shape, _log_int(rng, 1, 8192), rng.choice([0.0, 0.0, 0.5, 1.2]))


# ---- inputs ---------------------------------------------------------------------------------------

def _whole(rows):
    """What a program holds of rows (tokens, or a matrix's output channels): 8-bit integers and scales."""
    scale = (rows.abs().amax(-1) / 127).clamp(min=1e-30)
    return torch.round(rows / scale[..., None]).to(torch.int8), scale


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _tokens(gen, R, d):
    """Activations as products see them: a few channels far larger than the rest."""
    x = _randn(gen, R, d)
    x[:, torch.randperm(d, generator=gen, device="cuda")[:max(1, d // 256)]] *= 8
    return x


def _matrices(gen, E, N, K):
    q = torch.empty((E, N, K), dtype=torch.int8, device="cuda")
    scale = torch.empty((E, N), device="cuda")
    for e in range(E):
        q[e], scale[e] = _whole(_randn(gen, N, K) * 0.02)
    return q, scale


def _groups(gen, T, E, k, skew):
    """Row counts of E experts when each of T tokens picks k of them: offsets on the GPU, largest group."""
    load = torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32)) * -skew
    load = load[torch.randperm(E, generator=gen, device="cuda")]
    u = torch.rand((T, E), generator=gen, device="cuda").clamp(min=1e-20)
    picked = (load - torch.log(-torch.log(u))).topk(k, dim=1).indices
    counts = torch.bincount(picked.flatten(), minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    return offsets, int(counts.max())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed % 1000003)
    s, T = {"case": case}, case["T"]
    if case["op"] == "norm":
        d = case["d"]
        s["x"] = _randn(gen, T, d + case["gap"]).to(torch.bfloat16)[:, :d]
        residual = _tokens(gen, T, d) * 3
        kind = {"none": None, "bf16": torch.bfloat16, "fp32": torch.float32}[case["residual"]]
        s["residual"] = residual.to(kind) if kind else None
        s["weight"] = (1 + 0.1 * _randn(gen, d)).to(torch.bfloat16)
        if own:
            s["h"] = torch.empty_like(s["residual"]) if kind else None
            s["y"] = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
            s["q"] = torch.empty((T, d), dtype=torch.int8, device="cuda")
            s["scale"] = torch.empty(T, dtype=torch.float32, device="cuda")
        return s
    if case["op"] == "gemm":
        E, K, N = case["E"], case["K"], case["N"]
        s["offsets"], s["most"] = _groups(gen, T, E, 1, 0.0)
        s["x"], s["x_scale"] = _whole(_tokens(gen, T, K))
        s["w"], s["w_scale"] = _matrices(gen, E, N, K)
        rows, columns, out = T, N, torch.float32 if case["out"] == "fp32" else torch.bfloat16
        shape = (T, 512, 128, E, 1)
    else:
        d, f, E, k = (case[n] for n in ("d_model", "d_ff", "E", "k"))
        s["offsets"], s["most"] = _groups(gen, T, E, k, case["skew"])
        s["x"], s["x_scale"] = _whole(_tokens(gen, T * k, d))
        for name, n, m in (("w1", f, d), ("w3", f, d), ("w2", d, f)):
            s[name], s[name + "_scale"] = _matrices(gen, E, n, m)
        rows, columns, out = T * k, d, torch.bfloat16
        shape = (T, d, f, E, k)
    if own:
        from paper_2605_17889_amd import binding as B
        s["ctx"] = B.MoeContext(*shape)
        s["out"] = torch.empty((rows, columns), dtype=out, device="cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------

def _rows_in_8_bits(y):
    scale = y.abs().amax(-1) / 127
    q = torch.round(y / torch.where(scale > 0, scale, 1.0)[:, None])
    return torch.where(scale[:, None] > 0, q, 0.0), scale


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["weight"].float()
    q, scale = _rows_in_8_bits(y)
    return {"h": None if s["residual"] is None else h.to(s["residual"].dtype), "y": y.to(torch.bfloat16),
            "q": q.to(torch.bfloat16), "scale": scale}


def _by_expert(offsets, most):
    """[E, most] row of the padded batch's places, and which of them hold one."""
    at = torch.arange(most, device=offsets.device)
    first, count = offsets[:-1, None], (offsets[1:] - offsets[:-1])[:, None]
    held = at[None, :] < count
    return torch.where(held, first + at[None, :], 0), held


def _product(x, x_scale, w, w_scale):
    """[E, M, K] x [E, N, K] of whole numbers held in fp32, times the scales."""
    return torch.bmm(x, w.float().transpose(1, 2)) * x_scale[:, :, None] * w_scale[:, None, :]


def _plain_gemm(s):
    rows, held = _by_expert(s["offsets"], s["most"])
    y = _product(s["x"][rows].float(), s["x_scale"][rows], s["w"], s["w_scale"])
    return y[held].to(torch.float32 if s["case"]["out"] == "fp32" else torch.bfloat16)


def _plain_experts(s):
    rows, held = _by_expert(s["offsets"], s["most"])
    x, x_scale = s["x"][rows].float(), s["x_scale"][rows]
    gate = _product(x, x_scale, s["w1"], s["w1_scale"])
    up = _product(x, x_scale, s["w3"], s["w3_scale"])
    hidden = (gate / (1 + torch.exp(-gate)) * up).to(torch.bfloat16).float()   # H is a bf16 tensor by definition
    q, scale = _rows_in_8_bits(hidden.flatten(0, 1))
    y = _product(q.view(hidden.shape), scale.view(hidden.shape[:2]), s["w2"], s["w2_scale"])
    return y[held].to(torch.bfloat16)


def run(s):
    case = s["case"]
    if not own:
        return {"norm": _plain_norm, "gemm": _plain_gemm, "experts": _plain_experts}[case["op"]](s)
    from paper_2605_17889_amd import binding as B
    if case["op"] == "norm":
        B.moe_rmsnorm_i8(s["x"], s["residual"], s["weight"], EPS, s["h"], s["y"], s["q"], s["scale"])
        return {"h": s["h"], "y": s["y"], "q": s["q"].to(torch.bfloat16), "scale": s["scale"]}
    if case["op"] == "gemm":
        offsets = None if case["E"] == 1 else s["offsets"]
        B.moe_gemm_i8(s["ctx"], s["x"], s["x_scale"], offsets, case["T"], case["E"], case["N"], case["K"],
                      s["w"], s["w_scale"], s["out"])
        return s["out"]
    B.moe_expert_ffn_i8(s["ctx"], s["x"], s["x_scale"], s["offsets"], case["T"] * case["k"], s["w1"],
                        s["w1_scale"], s["w3"], s["w3_scale"], s["w2"], s["w2_scale"], s["out"])
    return s["out"]


def work(case):
    T = case["T"]
    if case["op"] == "norm":
        d = case["d"]
        stream = {"none": 0, "bf16": 2, "fp32": 4}[case["residual"]]
        return {"bytes": T * (d * (2 + 2 * stream + 2 + 1) + 4) + 2 * d, "flops": 10 * T * d}
    # experts that hold a row, under uniform picks
    touched = lambda E, k: E * (1.0 - (1.0 - k / E) ** T)
    if case["op"] == "gemm":
        K, N, E = case["K"], case["N"], case["E"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": touched(E, 1) * N * (K + 4) + T * (K + 4 + out * N), "flops": 2 * T * N * K}
    d, f, E, k = (case[n] for n in ("d_model", "d_ff", "E", "k"))
    weights = 3 * d * f + 4 * (2 * f + d)
    return {"bytes": touched(E, k) * weights + T * k * (d + 4 + 2 * d), "flops": 6 * T * k * d * f}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_rows_in_8_bits(y):
    peak = y.abs().max(dim=1, keepdim=True).values
    return torch.where(peak > 0, (y * 127 / peak).round(), torch.zeros_like(y)), peak[:, 0] / 127


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h += s["residual"].double()
        root = torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / case["d"] + EPS)
        y = h / root[:, None] * s["weight"].double()
        q, scale = _exact_rows_in_8_bits(y)
        return {"h": None if s["residual"] is None else h, "y": y, "q": q, "scale": scale}
    at = s["offsets"].tolist()
    experts = [(e, slice(at[e], at[e + 1])) for e in range(case["E"])]

    def times(x, scale, w, e):
        return (x @ s[w][e].double().t()) * (scale[:, None] * s[w + "_scale"][e].double()[None, :])

    columns = case["N"] if case["op"] == "gemm" else case["d_model"]
    y = torch.empty((at[-1], columns), dtype=torch.float64, device="cuda")
    for e, rows in experts:
        x, scale = s["x"][rows].double(), s["x_scale"][rows].double()
        if case["op"] == "gemm":
            y[rows] = times(x, scale, "w", e)
        elif rows.stop > rows.start:
            gate = times(x, scale, "w1", e)
            hidden = gate * torch.sigmoid(gate) * times(x, scale, "w3", e)
            y[rows] = times(*_exact_rows_in_8_bits(hidden.to(torch.bfloat16).double()), "w2", e)
    return y
