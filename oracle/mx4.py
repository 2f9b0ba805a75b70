"""Microscaled 4-bit floating point and routers by scores, in 64 bits from their definitions (test infrastructure)."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def runs(K: int) -> int:
    return -(-K // 256)


def arrange(scale: np.ndarray) -> np.ndarray:
    """[rows, blocks] bytes in the order of the blocks -> [runs, rows, 8], block 4t+g of a run at byte 2g+t."""
    rows, blocks = scale.shape
    out = np.zeros((runs(32 * blocks), rows, 8), np.uint8)
    for b in range(blocks):
        out[b // 8, :, 2 * (b % 4) + b % 8 // 4] = scale[:, b]
    return out


def by_block(arranged: np.ndarray, blocks: int) -> np.ndarray:
    return np.stack([arranged[b // 8, :, 2 * (b % 4) + b % 8 // 4] for b in range(blocks)], axis=1)


def codes_of(u: np.ndarray) -> np.ndarray:
    """Nearest codes (0..7) of |u|, ties to the even code; above 6: 7."""
    m = np.abs(u)
    code = np.zeros(m.shape, np.uint8)
    for c, tie in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (m > tie) if c % 2 == 0 else (m >= tie)
    return code


def scale_bytes(peak: np.ndarray) -> np.ndarray:
    """Of blocks whose largest |element| is `peak`: floor(log2) - 2 + 127, 0 at least; 255 where it is not finite."""
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(np.where(np.isfinite(peak), peak, 1.0))
    byte = np.where(peak == 0, 0, np.maximum(e - 1 - 2 + 127, 0))
    return np.where(np.isfinite(peak), byte, 255).astype(np.uint8)


def quantize(x: np.ndarray):
    """[rows, K] -> codes [rows, K/2], scales by block [rows, K/32]."""
    rows, K = x.shape
    blocks = x.astype(np.float64).reshape(rows, K // 32, 32)
    with np.errstate(invalid="ignore"):
        peak = np.where(np.isfinite(blocks).all(-1), np.abs(blocks).max(-1), np.inf)
    scale = scale_bytes(peak)
    fine = scale[..., None] != 255
    with np.errstate(invalid="ignore", over="ignore"):
        u = np.where(fine, np.ldexp(np.where(fine, blocks, 0.0), 127 - scale.astype(np.int64)[..., None]), 0.0)
    code = codes_of(u) | (8 * (np.signbit(u) & fine)).astype(np.uint8)
    code = code.reshape(rows, K)
    return code[:, 0::2] | code[:, 1::2] << 4, scale


def decode(q: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """codes [rows, K/2], scales by block -> numbers [rows, K]."""
    code = np.stack((q & 15, q >> 4), axis=-1).reshape(q.shape[0], -1)
    v = VALUES[code & 7] * np.where(code & 8, -1.0, 1.0)
    v = np.ldexp(v.reshape(q.shape[0], -1, 32), scale.astype(np.int64)[..., None] - 127)
    return np.where(scale[..., None] == 255, np.nan, v).reshape(code.shape)


def silu(g: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g))


def route(logits, correction, k, score="sigmoid", groups=1, top_groups=1, group_best=2, renormalise=True, scale=1.0):
    """Selection and weights of moe_route_scored with scores in fp32 (whose ties count, and whose exp(-l) is infinite past the
    largest fp32 number: a sigmoid of 0) and weights in 64 bits."""
    T, E = logits.shape
    l = np.where(np.isnan(logits), -np.inf, logits).astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            e = np.exp(-l)
            s = 1 / (1 + np.where(e > np.finfo(np.float32).max, np.inf, e))
        else:
            top = l.max(1, keepdims=True)
            e = np.where(l == top, 1.0, np.exp(l - top))
            s = e / e.sum(1, keepdims=True)
        c = s.astype(np.float32)
        if correction is not None:
            c = (c + correction.astype(np.float32)).astype(np.float32)
        c = np.where(np.isnan(c), -np.inf, c).astype(np.float64)
        size = E // groups
        idx = np.empty((T, k), np.int32)
        for t in range(T):
            best = np.sort(c[t].reshape(groups, size), axis=1)[:, ::-1][:, :group_best].sum(1)
            best = np.where(np.isnan(best), -np.inf, best)
            kept = np.argsort(-best, kind="stable")[:top_groups]
            allowed = np.concatenate([np.arange(g * size, (g + 1) * size) for g in np.sort(kept)])
            idx[t] = allowed[np.argsort(-c[t, allowed], kind="stable")[:k]]
    w = np.take_along_axis(s, idx.astype(np.int64), 1)
    if renormalise:
        total = w.sum(1, keepdims=True)
        w = np.where(total > 0, w / np.where(total > 0, total, 1), 0.0)
    return idx, w * scale
