"""The oracle of the 4-bit path and of routers by scores (oracle/mx4.py) against hand values and brute force."""
import numpy as np
import pytest

from oracle import mx4 as M


def test_codes_are_the_nearest_and_ties_go_to_even():
    u = np.unique(np.concatenate([np.linspace(0, 8, 4001), (M.VALUES[1:] + M.VALUES[:-1]) / 2]))
    for x in u:
        d = np.abs(M.VALUES - x)
        best = np.flatnonzero(d == d.min())
        want = best[0] if len(best) == 1 else best[best % 2 == 0][0]
        assert M.codes_of(np.array([x]))[0] == want and M.codes_of(np.array([-x]))[0] == want


def test_scales():
    peak = np.array([0.0, 1.0, 1.99, 2.0, 3.0, 4.0, 7.9, 8.0, 2.0 ** -125, 2.0 ** -126, 2.0 ** -133, 2.0 ** 127, np.inf, np.nan])
    assert M.scale_bytes(peak).tolist() == [0, 125, 125, 126, 126, 127, 127, 128, 0, 0, 0, 252, 255, 255]


def test_a_block_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [6.0, -7.9, 0.25, 0.75, -1.25, 5.0]            # scale 1: 6, -6 (saturated), 0, 1, -1, 4
    q, s = M.quantize(x)
    assert s.tolist() == [[127]] and q[0, :3].tolist() == [7 | 15 << 4, 0 | 2 << 4, 10 | 6 << 4] and not q[0, 3:].any()
    assert M.decode(q, s)[0, :6].tolist() == [6.0, -6.0, 0.0, 1.0, -1.0, 4.0]
    x[0, 9] = np.nan
    q, s = M.quantize(x)
    assert s.tolist() == [[255]] and not q.any() and np.isnan(M.decode(q, s)).all()


@pytest.mark.parametrize("blocks", [1, 3, 8, 9, 44])
def test_scales_are_arranged_by_runs(blocks):
    s = np.arange(5 * blocks, dtype=np.uint8).reshape(5, blocks) + 1
    a = M.arrange(s)
    assert a.shape == (M.runs(32 * blocks), 5, 8) and np.array_equal(M.by_block(a, blocks), s)
    padded = np.zeros((5, -(-blocks // 8) * 8), np.uint8)
    padded[:, :blocks] = s
    assert np.array_equal(a, padded.reshape(5, -1, 2, 4).transpose(1, 0, 3, 2).reshape(-1, 5, 8))


def test_routes_by_hand():
    logits = np.array([[0.0, 2.0, 1.0, -1.0, 3.0, 0.0, 0.0, 0.0]], np.float32)
    sig = lambda v: 1 / (1 + np.exp(-np.array(v, np.float64)))
    idx, w = M.route(logits, None, 2)
    assert idx.tolist() == [[4, 1]] and np.allclose(w[0], sig([3.0, 2.0]) / sig([3.0, 2.0]).sum())
    # two groups of four, each worth its two largest: 0.88 + 0.73 against 0.95 + 0.5
    idx, w = M.route(logits, None, 2, groups=2, top_groups=1, group_best=2, renormalise=False, scale=2.0)
    assert idx.tolist() == [[1, 2]] and np.allclose(w[0], 2 * sig([2.0, 1.0]))
    idx, _ = M.route(logits, None, 2, groups=2, top_groups=1, group_best=1)
    assert idx.tolist() == [[4, 5]]                             # worth its largest; then the first of the equal ones
    correction = np.array([0, 0, 0, 1.0, 0, 0, 0, 0], np.float32)
    idx, w = M.route(logits, correction, 1, score="softmax", renormalise=False)
    assert idx.tolist() == [[3]] and np.isclose(w[0, 0], np.exp(-1.0) / np.exp(logits.astype(np.float64)).sum())
