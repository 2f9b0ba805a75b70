"""Operators of the 4-bit path of a Mixture-of-Experts block and the router of layers with many experts, as a
program that serves such blocks calls them:

  route    experts of each token from router logits: scores (sigmoid, or softmax over all experts), a correction for
           balance that takes part in the choice only, the best groups of experts, the best experts in them, weights
           (moe_route_scored_from_logits)
  rows     rows of bf16 in microscaled 4-bit floating point, blocks of 32 elements with a power of two each, and back
           (moe_quantize_mx4, moe_dequantize_mx4)
  gemm     matrix product of such operands, one matrix or one per expert over rows grouped by expert (moe_gemm_mx4)
  experts  the gated feed-forward network of all experts over such rows grouped by expert (moe_expert_ffn_mx4): two
           products, SiLU(gate) * up brought to 4 bits again block by block, as the operator is defined, the third product

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


def _route(T, E, k, score="sigmoid", groups=1, top_groups=1, group_best=2, correction=True, renormalise=True,
           scale=2.5):
    return {"op": "route", "T": T, "E": E, "k": k, "score": score,
            "groups": groups, "top_groups": top_groups,   # equal ranges of experts; how many of them a token may use
            "group_best": group_best,                     # a group counts as much as its best expert, or its two best
            "correction": correction, "renormalise": renormalise, "scale": scale}


def _rows(T, d, gap=0):
    return {"op": "rows", "T": T, "d": d,
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
        # decode of a single sequence through a router of 256 experts in 8 groups: all latency
        named("route_t1_e256_groups", _route(1, 256, 8, groups=8, top_groups=4)),
        # a ragged prefill chunk through 64 experts, softmax over all of them, weights as they are
        named("route_t5003_e64_softmax", _route(5003, 64, 6, score="softmax", correction=False, renormalise=False, scale=1.0)),
        # a prefill chunk through the router of 256 experts
        named("route_t8192_e256_groups", _route(8192, 256, 8, groups=8, top_groups=4)),
        # a ragged batch of an odd number of blocks, rows cut out of a wider tensor
        named("rows_t1003_d1120_strided", _rows(1003, 1120, gap=37)),
        # the headline prefill chunk
        named("rows_t8192_d6144", _rows(8192, 6144)),
        # decode of a single sequence through one projection with a long reduction: weights stream by
        named("gemm_t1_k14336_n4096", _gemm(1, 14336, 4096)),
        # a ragged decode batch through a wide matrix, fp32 outputs (logits of a head)
        named("gemm_t37_k2048_n32000_fp32", _gemm(37, 2048, 32000, out="fp32")),
        # the headline prefill chunk through one dense projection
        named("gemm_t8192_k6144_n16384", _gemm(8192, 6144, 16384)),
        # decode of a single sequence: eight of 128 experts hold a row, all other groups are empty
        named("experts_qwen3_t1", _experts("qwen3_30b_a3b", 1)),
        # batched decode through large experts: all weights are read for a handful of rows each
        named("experts_mixtral8x7b_t16", _experts("mixtral8x7b", 16)),
        # prefill of a ragged number of tokens through many small experts, loads as skewed as routers skew them, a
        # reduction that is no multiple of 256
        named("experts_deepseek_v2_lite_t5003_skewed", _experts("deepseek_v2_lite", 5003, skew=0.5)),
        # the headline prefill chunk
        named("experts_mixtral8x22b_t8192", _experts("mixtral8x22b", 8192)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "rows", "gemm", "gemm", "experts", "experts"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        size = rng.randint(2, 256 // groups)
        top_groups = rng.randint(1, groups)
        k = _log_int(rng, 1, min(16, top_groups * size))
        return _route(_log_int(rng, 1, 16384), groups * size, k, rng.choice(["sigmoid", "softmax"]), groups, top_groups,
                      rng.randint(1, 2), rng.random() < 0.7, rng.random() < 0.7, rng.choice([1.0, 2.5]))
    if op == "rows":
        d = 32 * _log_int(rng, 1, 512)
        T = min(_log_int(rng, 1, 16384), (8192 * 6144) // d)
        return _rows(T, d, rng.choice([0, 0, rng.randint(1, 512)]))
    if op == "gemm":
        E = rng.choice([1, 1, 1, rng.randint(2, 32)])
        K = 32 * _log_int(rng, 4, 512)
        N = 16 * _log_int(rng, 4, 2048 if E == 1 else 256)
        T = min(_log_int(rng, 1, 8192), int(8192 * 6144 * 16384 / (K * N)))
        return _gemm(T, K, N, E, rng.choice(["bf16", "bf16", "fp32"]))
    shape = rng.choice(sorted(SHAPES))
    return _experts(shape, _log_int(rng, 1, 8192), rng.choice([0.0, 0.0, 0.5, 1.2]))


# ---- inputs ---------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _arranged(scale):
    """Scales of blocks [rows, blocks] as the operators hold them: 8 blocks (256 elements) of a row side by side,
    block 4 * t + g of them at 2 * g + t; 0 behind the last block."""
    rows, blocks = scale.shape
    whole = torch.zeros((rows, -(-blocks // 8) * 8), dtype=torch.uint8, device=scale.device)
    whole[:, :blocks] = scale
    return whole.view(rows, -1, 2, 4).permute(1, 0, 3, 2).reshape(-1, rows, 8).contiguous()


def _packed(rows):
    """What a program holds of rows (tokens, or a matrix's output channels): two elements to a byte, arranged scales."""
    blocks = rows.view(rows.shape[0], -1, 32)
    power = torch.frexp(blocks.abs().amax(-1)).exponent - 3
    u = torch.ldexp(blocks, -power[..., None])
    code = torch.bucketize(u.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=rows.device))
    code = (code + 8 * (u < 0)).to(torch.uint8).view(rows.shape[0], -1, 2)
    return code[..., 0] | code[..., 1] << 4, _arranged((power + 127).to(torch.uint8))


def _tokens(gen, R, d):
    """Activations as products see them: a few channels far larger than the rest."""
    x = _randn(gen, R, d)
    x[:, torch.randperm(d, generator=gen, device="cuda")[:max(1, d // 256)]] *= 8
    return x


def _matrices(gen, E, N, K):
    q = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    scale = torch.empty((E, -(-K // 256), N, 8), dtype=torch.uint8, device="cuda")
    for e in range(E):
        q[e], scale[e] = _packed(_randn(gen, N, K) * 0.02)
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


def _logits(gen, case, correction):
    """Router logits whose choices do not hang on the last bits of a score: tokens with two that are closer than that
    where the choice is made are drawn again."""
    T, E, k, G = (case[n] for n in ("T", "E", "k", "groups"))
    logits = _randn(gen, T, E) * 1.5
    for _ in range(50):
        score = logits.double()
        score = torch.sigmoid(score) if case["score"] == "sigmoid" else torch.softmax(score, 1)
        if correction is not None:
            score = score + correction.double()
        part = score.view(T, G, -1)
        value = part.topk(min(case["group_best"], E // G), dim=2).values.sum(2)
        near = torch.zeros(T, dtype=torch.bool, device="cuda")
        if G > case["top_groups"]:
            order = value.sort(1, descending=True).values
            last = order[:, case["top_groups"] - 1]
            near |= last - order[:, case["top_groups"]] < 1e-5 * last.abs()
            allowed = value >= last[:, None]
            score = torch.where(allowed[:, :, None], part, -math.inf).flatten(1)
        best = score.sort(1, descending=True).values[:, :k + 1]
        near |= (best[:, :-1] - best[:, 1:] < 1e-5 * best[:, :-1].abs()).any(1)
        if not bool(near.any()):
            break
        logits = torch.where(near[:, None], _randn(gen, T, E) * 1.5, logits)
    return logits


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed % 1000003)
    s, T = {"case": case}, case["T"]
    if case["op"] == "route":
        E, k = case["E"], case["k"]
        s["correction"] = _randn(gen, E) * 0.05 if case["correction"] else None
        s["logits"] = _logits(gen, case, s["correction"])
        if own:
            from paper_2605_17889_amd import binding as B
            s["ctx"] = B.MoeContext(T, 512, 128, E, k)
            s["scoring"] = B.MoeScoring(case["score"], groups=case["groups"], top_groups=case["top_groups"],
                                        group_best=case["group_best"], renormalise=case["renormalise"], scale=case["scale"])
            s["idx"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
            s["weight"] = torch.empty((T, k), dtype=torch.float32, device="cuda")
        return s
    if case["op"] == "rows":
        d = case["d"]
        s["x"] = _tokens(gen, T, d + case["gap"]).to(torch.bfloat16)[:, :d]
        if own:
            s["q"] = torch.empty((T, d // 2), dtype=torch.uint8, device="cuda")
            s["scale"] = torch.empty((-(-d // 256), T, 8), dtype=torch.uint8, device="cuda")
            s["y"] = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
        return s
    if case["op"] == "gemm":
        E, K, N = case["E"], case["K"], case["N"]
        s["offsets"], s["most"] = _groups(gen, T, E, 1, 0.0)
        s["x"], s["x_scale"] = _packed(_tokens(gen, T, K))
        s["w"], s["w_scale"] = _matrices(gen, E, N, K)
        rows, columns, out = T, N, torch.float32 if case["out"] == "fp32" else torch.bfloat16
        shape = (T, 512, 128, E, 1)
    else:
        d, f, E, k = (case[n] for n in ("d_model", "d_ff", "E", "k"))
        s["offsets"], s["most"] = _groups(gen, T, E, k, case["skew"])
        s["x"], s["x_scale"] = _packed(_tokens(gen, T * k, d))
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

def _plain_route(s):
    case = s["case"]
    T, E, k, G = (case[n] for n in ("T", "E", "k", "groups"))
    logits = s["logits"]
    if case["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-logits))
    else:
        e = torch.exp(logits - logits.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    choice = score if s["correction"] is None else score + s["correction"]
    if G > case["top_groups"]:
        part = choice.view(T, G, -1)
        value = part.sort(dim=2, descending=True, stable=True).values[:, :, :case["group_best"]].sum(2)
        rank = value.sort(dim=1, descending=True, stable=True).indices.argsort(1)
        choice = torch.where((rank < case["top_groups"])[:, :, None], part, -math.inf).flatten(1)
    idx = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    weight = score.gather(1, idx)
    if case["renormalise"]:
        weight = weight / weight.sum(1, keepdim=True)
    return {"idx": idx.to(torch.int32), "weight": weight * case["scale"]}


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _in_4_bits(v):
    """fp32 [rows, K] -> the multiples of their blocks' powers of two that stand for them, and the powers."""
    blocks = v.view(v.shape[0], -1, 32)
    power = (torch.frexp(blocks.abs().amax(-1)).exponent - 3).clamp(min=-127)
    u = torch.ldexp(blocks, -power[..., None])
    m = u.abs()
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))
    value = torch.tensor(_VALUES, device=v.device)[code.int()]
    return torch.where(u < 0, -value, value), power


def _numbers(q, scale):
    """Packed rows [.., rows, K / 2] and arranged scales [.., chunks, rows, 8] as the fp32 numbers they stand for."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=q.device)
    v = table[torch.stack((q & 15, q >> 4), dim=-1).int()].flatten(-2)
    K = v.shape[-1]
    lead = scale.shape[:-3]
    by_block = scale.view(*lead, *scale.shape[-3:-1], 4, 2).transpose(-1, -2).movedim(-4, -3).reshape(*v.shape[:-1], -1)
    power = by_block[..., :K // 32].to(torch.int32) - 127
    return torch.ldexp(v.view(*v.shape[:-1], -1, 32), power[..., None]).flatten(-2)


def _plain_rows(s):
    value, power = _in_4_bits(s["x"].float())
    return torch.ldexp(value, power[..., None]).flatten(1).to(torch.bfloat16)


def _by_expert(offsets, most):
    """[E, most] row of the padded batch's places, and which of them hold one."""
    at = torch.arange(most, device=offsets.device)
    first, count = offsets[:-1, None], (offsets[1:] - offsets[:-1])[:, None]
    held = at[None, :] < count
    return torch.where(held, first + at[None, :], 0), held


def _plain_gemm(s):
    rows, held = _by_expert(s["offsets"], s["most"])
    x = _numbers(s["x"], s["x_scale"])[rows]
    y = torch.bmm(x, _numbers(s["w"], s["w_scale"]).transpose(1, 2))
    return y[held].to(torch.float32 if s["case"]["out"] == "fp32" else torch.bfloat16)


def _plain_experts(s):
    rows, held = _by_expert(s["offsets"], s["most"])
    x = _numbers(s["x"], s["x_scale"])[rows]
    gate = torch.bmm(x, _numbers(s["w1"], s["w1_scale"]).transpose(1, 2))
    up = torch.bmm(x, _numbers(s["w3"], s["w3_scale"]).transpose(1, 2))
    hidden = gate / (1 + torch.exp(-gate)) * up
    value, power = _in_4_bits(hidden.flatten(0, 1))
    h = torch.ldexp(value, power[..., None]).view(hidden.shape)
    return torch.bmm(h, _numbers(s["w2"], s["w2_scale"]).transpose(1, 2))[held].to(torch.bfloat16)


def run(s):
    case = s["case"]
    if not own:
        return {"route": _plain_route, "rows": _plain_rows, "gemm": _plain_gemm, "experts": _plain_experts}[case["op"]](s)
    from paper_2605_17889_amd import binding as B
    if case["op"] == "route":
        B.moe_route_scored_from_logits(s["ctx"], s["logits"], s["correction"], s["scoring"], case["T"], s["idx"], s["weight"])
        return {"idx": s["idx"], "weight": s["weight"]}
    if case["op"] == "rows":
        B.moe_quantize_mx4(s["x"], s["q"], s["scale"])
        B.moe_dequantize_mx4(s["q"], s["scale"], s["y"])
        return s["y"]
    if case["op"] == "gemm":
        offsets = None if case["E"] == 1 else s["offsets"]
        B.moe_gemm_mx4(s["ctx"], s["x"], s["x_scale"], offsets, case["T"], case["E"], case["N"], case["K"], s["w"],
                       s["w_scale"], s["out"])
        return s["out"]
    B.moe_expert_ffn_mx4(s["ctx"], s["x"], s["x_scale"], s["offsets"], case["T"] * case["k"], s["w1"], s["w1_scale"],
                         s["w3"], s["w3_scale"], s["w2"], s["w2_scale"], s["out"])
    return s["out"]


def work(case):
    T = case["T"]
    if case["op"] == "route":
        return {"bytes": 4 * T * case["E"] + 8 * T * case["k"], "flops": 10 * T * case["E"]}
    packed = lambda rows, K: rows * (K / 2 + K / 32)
    if case["op"] == "rows":
        return {"bytes": 2 * T * case["d"] + packed(T, case["d"]) + 2 * T * case["d"], "flops": 4 * T * case["d"]}
    # experts that hold a row, under uniform picks
    touched = lambda E, k: E * (1.0 - (1.0 - k / E) ** T)
    if case["op"] == "gemm":
        K, N, E = case["K"], case["N"], case["E"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": packed(touched(E, 1) * N, K) + packed(T, K) + T * out * N, "flops": 2 * T * N * K}
    d, f, E, k = (case[n] for n in ("d_model", "d_ff", "E", "k"))
    return {"bytes": touched(E, k) * 3 * packed(f, d) + T * k * 2 * d + packed(T * k, d), "flops": 6 * T * k * d * f}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _decoded(q, scale):
    """One matrix of packed rows and its arranged scales as numbers in 64 bits, bit by bit from the format: sign, two bits
    of exponent (bias 1), one bit of fraction; an exponent of 0 has no leading one."""
    code = torch.empty((q.shape[0], 2 * q.shape[1]), dtype=torch.int64, device=q.device)
    code[:, 0::2], code[:, 1::2] = (q & 15).long(), (q >> 4).long()
    exponent, fraction = (code >> 1) & 3, (code & 1).double()
    value = torch.where(exponent == 0, fraction / 2, (1 + fraction / 2) * torch.pow(2.0, (exponent - 1).double()))
    value = torch.where(code >= 8, -value, value)
    block = torch.arange(value.shape[1], device=q.device) // 32
    byte = scale[block // 8, :, 2 * (block % 4) + block % 8 // 4].t()
    return value * torch.pow(2.0, byte.double() - 127)


def _exact_in_4_bits(v):
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=v.device)
    middles = (grid[1:] + grid[:-1]) / 2
    blocks = v.reshape(v.shape[0], -1, 32)
    unit = torch.pow(2.0, torch.floor(torch.log2(blocks.abs().amax(2, keepdim=True).clamp(min=2.0 ** -125))) - 2)
    u = blocks.abs() / unit
    below = torch.bucketize(u, middles)                         # a middle belongs to the value below it
    tie = torch.isin(u, middles) & (below % 2 == 1)             # unless the one above has the even code
    return (torch.sign(blocks) * grid[(below + tie).clamp(max=7)] * unit).reshape(v.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        l = s["logits"].double()
        score = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l, dim=1)
        choice = score.clone() if s["correction"] is None else score + s["correction"].double()
        size = case["E"] // case["groups"]
        if case["top_groups"] < case["groups"]:
            value = torch.stack([choice[:, g * size:(g + 1) * size].topk(min(case["group_best"], size), dim=1).values.sum(1)
                                 for g in range(case["groups"])], dim=1)
            keep = torch.zeros_like(value).scatter_(1, value.topk(case["top_groups"], dim=1).indices, 1.0)
            choice[keep.repeat_interleave(size, dim=1) == 0] = -math.inf
        idx = choice.topk(case["k"], dim=1, sorted=True).indices
        weight = torch.take_along_dim(score, idx, 1)
        if case["renormalise"]:
            weight = weight / weight.sum(dim=1, keepdim=True)
        return {"idx": idx.to(torch.int32), "weight": weight * case["scale"]}
    if case["op"] == "rows":
        return _exact_in_4_bits(s["x"].double())
    at = s["offsets"].tolist()
    x = _decoded(s["x"], s["x_scale"])
    columns = case["N"] if case["op"] == "gemm" else case["d_model"]
    y = torch.empty((at[-1], columns), dtype=torch.float64, device="cuda")
    for e in range(case["E"]):
        rows = slice(at[e], at[e + 1])
        if rows.start == rows.stop:
            continue
        times = lambda v, w: v @ _decoded(s[w][e], s[w + "_scale"][e]).t()
        if case["op"] == "gemm":
            y[rows] = times(x[rows], "w")
        else:
            gate = times(x[rows], "w1")
            y[rows] = times(_exact_in_4_bits(gate * torch.sigmoid(gate) * times(x[rows], "w3")), "w2")
    return y
