"""Pins for the oracle of rows in few bits and of the distillation loss: hand-computed codes and
losses, and properties fixed by the definitions (gradients against differences)."""
import math

import numpy as np
import pytest

from oracle import distill, mx


def test_magnitudes():
    assert mx.magnitudes(4) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert mx.magnitudes(6) == [i / 8 for i in range(16)] + [i / 4 for i in range(8, 16)] + [i / 2 for i in range(8, 16)]


@pytest.mark.parametrize("bits,x,scale,vals", [
    # amax 6 -> 2^0; ties to the even code: 0.25 -> 0, 0.75 -> 1, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    (4, [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, 0.26], 127, [6, 0, 1, 1, 2, 2, 4, 4, -6, 0.5]),
    # amax 7.9 saturates; amax 8 moves the scale
    (4, [7.9, -7, 1], 127, [6, -6, 1]),
    (4, [8, 7.9, 1], 128, [8, 8, 1]),
    (6, [7.5, 7.9, 0.0625, 0.1875, 2.125, 4.25, -3.9], 127, [7.5, 7.5, 0, 0.25, 2, 4, -4]),
    (6, [0.03, -0.001], 127 - 6 - 2, [7.5 / 256, -0.25 / 256]),
    (4, [0.0, -0.0], 0, [0, 0]),
    (4, [2.0 ** -126, 2.0 ** -127], 0, [2.0 ** -126, 2.0 ** -127]),
    (4, [1e-45, 0], 0, [0, 0]),
])
def test_quantize_by_hand(bits, x, scale, vals):
    codes, scales = mx.quantize(np.array([x], dtype=np.float64), bits)
    assert scales[0, 0] == scale
    np.testing.assert_array_equal(mx.values(codes, scales, len(x), bits)[0], vals)


def test_blocks_with_infinities_or_nans_are_nan():
    x = np.ones((1, 70))
    x[0, 3], x[0, 66] = np.inf, np.nan
    codes, scales = mx.quantize(x, 4)
    v = mx.values(codes, scales, 70, 4)[0]
    assert scales.tolist() == [[255, 125, 255]] and not codes[0, [0, 2]].any()
    assert np.isnan(v[:32]).all() and (v[32:64] == 1).all() and np.isnan(v[64:]).all()


@pytest.mark.parametrize("bits", [4, 6])
def test_pack_round_trip(bits):
    g = np.random.default_rng(3)
    c = g.integers(0, 1 << bits, size=(5, 3, 32))
    p = mx.pack(c, bits)
    assert p.shape == (5, 3, 4 * bits)
    np.testing.assert_array_equal(mx.unpack(p, bits), c)
    assert p[0, 0, 0] == (c[0, 0, 0] | c[0, 0, 1] << bits) & 255  # lowest bits first


@pytest.mark.parametrize("bits", [4, 6])
def test_quantize_is_nearest_and_idempotent(bits):
    g = np.random.default_rng(4)
    x = g.normal(size=(40, 65)) * 2.0 ** g.integers(-20, 20, size=(40, 65))
    c, s = mx.quantize(x, bits)
    v = mx.values(c, s, 65, bits)
    c2, s2 = mx.quantize(v, bits)
    np.testing.assert_array_equal(mx.values(c2, s2, 65, bits), v)
    step = 2.0 ** (s.astype(float) - 127).repeat(32, axis=1)[:, :65]
    assert (np.abs(v - x) <= (1.0 if bits == 4 else 0.25) * step + (np.abs(x) > 6 * step) * 2 * step).all()


def test_scores_grad_against_differences():
    g = np.random.default_rng(5)
    q, x, up = g.normal(size=(3, 8)), g.normal(size=(5, 8)), g.normal(size=(3, 5))
    f = lambda a, b: float((up * mx.scores(a, b)).sum())
    dq, dx = mx.scores_grad(up, x), mx.scores_grad(up, q, transposed=True)
    for base, grad, fn in ((q, dq, lambda a: f(a, x)), (x, dx, lambda b: f(q, b))):
        for i in np.ndindex(base.shape):
            e = np.zeros_like(base)
            e[i] = 1e-6
            assert abs((fn(base + e) - fn(base - e)) / 2e-6 - grad[i]) < 1e-7


def test_distill_by_hand():
    # two rows with logits 0 and ln 3 at temperature 1: student (1/4, 3/4); teacher: row 0 alone
    loss, lse, grad = distill.distill([[0.0, math.log(3)]], [[0, -1]], [[5.0, -math.inf]], 1.0, 1.0)
    assert abs(loss[0] - math.log(4)) < 1e-15 and abs(lse[0] - math.log(4)) < 1e-15
    np.testing.assert_allclose(grad, [[0.25 - 1, 0.75]], atol=1e-15)
    # teacher = student: no loss, no gradient; temperatures scale both sides
    loss, _, grad = distill.distill([[0.0, 2 * math.log(3)]], [[1, 0]], [[3 * math.log(3), 0.0]], 2.0, 3.0, [7.0])
    assert abs(loss[0]) < 1e-15 and np.abs(grad).max() < 1e-15
    # no entries: ids outside the rows, scores of -inf
    loss, lse, grad = distill.distill([[1.0, 2.0]], [[-1, 2, 0]], [[1.0, 1.0, -math.inf]], 1.0, 1.0)
    assert loss[0] == 0 and not grad.any() and np.isfinite(lse[0])
    # a masked row that the teacher wants; every row masked
    loss, _, grad = distill.distill([[0.0, -math.inf], [-math.inf] * 2], [[1], [0]], [[1.0], [1.0]], 1.0, 1.0)
    assert loss.tolist() == [math.inf, math.inf] and grad.tolist() == [[1.0, -1.0], [-1.0, 0.0]]


def test_distill_grad_against_differences():
    g = np.random.default_rng(6)
    s = g.normal(size=(4, 9))
    s[2, 4] = -np.inf
    ids = np.array([[0, 3, 8], [1, 1, -1], [7, 6, 5], [-1, -1, -1]])  # a repeated id, a short list, an empty one
    t = g.normal(size=(4, 3))
    w = g.uniform(0.5, 2, size=4)
    loss, _, grad = distill.distill(s, ids, t, 0.3, 0.7, w)
    for q, i in np.ndindex(s.shape):
        if not np.isfinite(s[q, i]):
            assert grad[q, i] == 0
            continue
        hi, lo = s.copy(), s.copy()
        hi[q, i] += 1e-5
        lo[q, i] -= 1e-5
        d = (distill.distill(hi, ids, t, 0.3, 0.7)[0] - distill.distill(lo, ids, t, 0.3, 0.7)[0]) / 2e-5
        assert abs(w[q] * d[q] - grad[q, i]) < 1e-7
        assert np.abs(np.delete(d, q)).max() == 0
