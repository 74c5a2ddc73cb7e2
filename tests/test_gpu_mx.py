"""Rows in few bits on the GPU (quantisation, values, products, the products' gradient) against the fp64 oracle.

Codes, scales and values are exact.  A product or a gradient element is a sum of K terms in fp32: it is held to
2 gamma_K sum |terms| (gamma_K = K 2^-24; K + 16 for short sums), plus the rounding of a 16-bit output."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import mx
from tests.gpu_helpers import DT, device, log

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 0.0, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


def draw(seed, n, d, dtype="f32", unit=True):
    g = np.random.default_rng(seed)
    x = g.normal(size=(n, d)).astype(np.float32)
    if unit and n:
        x /= np.linalg.norm(x, axis=1, keepdims=True)
    return torch.from_numpy(x).to(DT[dtype])


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def stored(r):
    """(codes, scales) of MxRows' rows, as the oracle has them."""
    c = r.codes.cpu().numpy()[r.first:r.first + r.n]
    s = r.scales.cpu().numpy()[r.first:r.first + r.n].astype(np.int64)
    return mx.unpack(c, r.bits), s


def make(seed, n, d, bits, dev):
    """Random codes and scales (every code; scales over 30 binades) as MxRows, and their fp64 values."""
    g = np.random.default_rng(seed)
    nb = (d + 31) // 32
    codes = g.integers(0, 1 << bits, size=(n, nb, 32))
    codes.reshape(n, -1)[:, d:] = 0
    scales = g.integers(105, 135, size=(n, nb))
    r = P.MxRows(torch.from_numpy(mx.pack(codes, bits)).to(dev), torch.from_numpy(scales.astype(np.uint8)).to(dev), d)
    return r, mx.values(codes, scales, d, bits)


def check_sums(got, want, absum, k, dtype, label):
    got, err = f64(got), np.abs(f64(got) - want)
    tol = 2 * (k + 16) * 2.0 ** -24 * absum + HALF_ULP[dtype] * 1.001 * np.abs(want) + SMALLEST[dtype]
    assert got.shape == want.shape
    assert np.isfinite(got).all(), label
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (label, worst, got[worst], want[worst], tol[worst])


# ------------------------------------------------------------------------------------- quantise, values
@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 1024), (3, 31), (2, 32), (5, 33), (67, 100), (9, 127), (300, 128), (17, 260),
                                 (4, 8192), (130, 384), (33, 1001), (1025, 8)])
def test_quantize_and_values_match_the_oracle(bits, dtype, n, d):
    dev = device()
    log("quantize", bits, dtype, n, d)
    x = draw(n * 131 + d, n, d, dtype, unit=d > 1)
    r = P.mx_quantize(x.to(dev), bits)
    want_c, want_s = mx.quantize(f64(x), bits)
    c, s = stored(r)
    np.testing.assert_array_equal(s, want_s)
    np.testing.assert_array_equal(c, want_c)
    want = mx.values(want_c, want_s, d, bits)
    for out in ("f32", "bf16", "f16"):
        got = P.mx_values(r, DT[out])
        ref = torch.from_numpy(want).to(DT[out])
        assert torch.equal(got.cpu(), ref), out
        assert torch.equal(torch.signbit(got.cpu()), torch.signbit(ref)), out


@pytest.mark.parametrize("bits", [4, 6])
def test_quantize_special_values(bits):
    dev = device()
    f = torch.finfo(torch.float32)
    x = torch.zeros((9, 64), dtype=torch.float32)
    x[0, 5], x[0, 40] = float("inf"), 1.0
    x[1, 0], x[1, 33] = float("nan"), -2.0
    x[2, :32], x[2, 32:] = f.max, -f.max
    x[3, :32] = torch.tensor([f.tiny, -f.tiny / 2, 2.0 ** -149, -(2.0 ** -149)] * 8)
    x[4, :] = -0.0
    x[5, :32] = 2.0 ** -126 * torch.arange(32) / 8
    x[6, :32] = torch.arange(32) / 4 - 4
    x[7, :] = torch.linspace(-7.99, 7.99, 64)
    x[8, 63] = -float("inf")
    r = P.mx_quantize(x.to(dev), bits)
    c, s = stored(r)
    want_c, want_s = mx.quantize(f64(x), bits)
    np.testing.assert_array_equal(s, want_s)
    np.testing.assert_array_equal(c, want_c)
    v = f64(P.mx_values(r))
    np.testing.assert_array_equal(v, mx.values(want_c, want_s, 64, bits))
    assert np.isnan(v[0, :32]).all() and (v[0, 32:] != 0).sum() == 1


@pytest.mark.parametrize("bits", [4, 6])
def test_every_code_under_every_scale_has_its_value(bits):
    dev = device()
    codes = np.tile(np.arange(1 << bits), 64 // (1 << bits) if bits == 4 else 1).reshape(1, 2, 32).repeat(256, axis=0)
    scales = np.arange(256).reshape(256, 1).repeat(2, axis=1)
    r = P.MxRows(torch.from_numpy(mx.pack(codes, bits)).to(dev), torch.from_numpy(scales.astype(np.uint8)).to(dev), 64)
    want = torch.from_numpy(mx.values(codes, scales, 64, bits))
    for out in ("f32", "bf16", "f16"):
        got = P.mx_values(r, DT[out]).cpu()
        ref = want.to(torch.float32).to(DT[out])  # fp32 holds every one
        assert torch.equal(got.nan_to_num(nan=123.0), ref.nan_to_num(nan=123.0)), out


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,ld", [(100, 104), (100, 101), (64, 67), (33, 160), (7, 9)])
def test_quantize_and_values_of_strided_rows(bits, dtype, d, ld):
    dev = device()
    log("strided", bits, dtype, d, ld)
    n = 37
    wide = draw(5, n, ld, dtype).to(dev)
    r = P.mx_quantize(wide[:, :d], bits)
    want_c, want_s = mx.quantize(f64(wide[:, :d]), bits)
    c, s = stored(r)
    np.testing.assert_array_equal(c, want_c)
    np.testing.assert_array_equal(s, want_s)
    out = torch.full((n, ld), 7.0, dtype=DT[dtype], device=dev)
    P.mx_values(r, DT[dtype], out=out[:, :d])
    assert torch.equal(out[:, :d].cpu(), torch.from_numpy(mx.values(c, s, d, bits)).to(DT[dtype]))
    assert (out[:, d:] == 7).all()


@pytest.mark.parametrize("bits", [4, 6])
def test_quantize_appends_into_a_part(bits):
    dev = device()
    d, n = 96, 50
    x = draw(11, n, d).to(dev)
    whole = P.mx_quantize(x, bits)
    r = P.MxRows.empty(n + 5, d, bits)
    r.codes.fill_(0xAB)
    r.scales.fill_(0xCD)
    for a, b in ((0, 1), (1, 18), (18, 18), (18, 50)):
        P.mx_quantize(x[a:b], bits, out=r.part(a, b - a))
    assert torch.equal(r.codes[:n], whole.codes) and torch.equal(r.scales[:n], whole.scales)
    assert (r.codes[n:] == 0xAB).all() and (r.scales[n:] == 0xCD).all()
    assert torch.equal(P.mx_values(r.part(7, 9)), P.mx_values(whole)[7:16])


def test_quantize_offsets_past_32_bits():
    dev = device()
    n, d = (1 << 22) + 3, 1024  # 2^32 elements and more
    x = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
    for a in range(0, n, 1 << 19):
        b = min(n, a + (1 << 19))
        x[a:b] = torch.randn((b - a, d), device=dev).to(torch.bfloat16)
    log("quantize", n, d)
    r = P.mx_quantize(x, 4)
    at = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, n - 1], device=dev)
    want_c, want_s = mx.quantize(f64(x[at]), 4)
    np.testing.assert_array_equal(mx.unpack(r.codes[at].cpu().numpy(), 4), want_c)
    np.testing.assert_array_equal(r.scales[at].cpu().numpy(), want_s)
    v = P.mx_values(r, torch.bfloat16, out=x)
    np.testing.assert_array_equal(f64(v[at]), mx.values(want_c, want_s, d, 4))
    q = r.part(n - 5, 5)  # codes of rows past 2 GiB
    s = P.mx_scores(q, r.part(n - 9, 9))
    want = mx.scores(f64(v[n - 5:]), f64(v[n - 9:]))
    check_sums(s, want, np.abs(f64(v[n - 5:])) @ np.abs(f64(v[n - 9:])).T, d, "f32", "far rows")


# ------------------------------------------------------------------------------------- products
SHAPES = [(1, 1, 1), (1, 300, 32), (2, 15, 33), (16, 16, 128), (17, 64, 100), (5, 1000, 384), (33, 129, 160), (64, 257, 256),
          (77, 515, 1024), (100, 31, 96), (128, 128, 512), (129, 640, 224), (3, 5000, 1024), (250, 400, 768), (1, 77, 8192),
          (40, 50, 8190), (513, 33, 64), (1, 4096, 1024), (16, 2049, 640), (600, 700, 416)]


@pytest.mark.parametrize("qb,rb", [(4, 4), (6, 4), (4, 6), (6, 6)])
@pytest.mark.parametrize("nq,n,d", SHAPES)
def test_scores_match_the_oracle(qb, rb, nq, n, d):
    dev = device()
    log("scores", qb, rb, nq, n, d)
    q, qv = make(nq + d, nq, d, qb, dev)
    r, rv = make(n + d, n, d, rb, dev)
    want, absum = mx.scores(qv, rv), np.abs(qv) @ np.abs(rv).T
    for dtype in ("f32", "bf16", "f16"):
        if dtype == "f16" and absum.max() > 6e4:
            scale = 2.0 ** -14
            r2 = P.MxRows(r.codes, r.scales - 14, d)
            check_sums(P.mx_scores(q, r2, DT[dtype]), want * scale, absum * scale, d, dtype, (dtype, nq, n, d))
        else:
            check_sums(P.mx_scores(q, r, DT[dtype]), want, absum, d, dtype, (dtype, nq, n, d))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad", [1, 2, 8, 16])
def test_scores_into_strided_rows_and_of_parts(dtype, pad):
    dev = device()
    nq, n, d = 37, 203, 160
    q, qv = make(1, nq + 4, d, 6, dev)
    r, rv = make(2, n + 9, d, 4, dev)
    wide = torch.full((nq, n + pad), 7.0, dtype=DT[dtype], device=dev)
    P.mx_scores(q.part(3, nq), MxScaled(r, -14).part(5, n), DT[dtype], out=wide[:, :n])
    f = 2.0 ** -14
    want, absum = mx.scores(qv[3:3 + nq], rv[5:5 + n]) * f, np.abs(qv[3:3 + nq]) @ np.abs(rv[5:5 + n]).T * f
    check_sums(wide[:, :n], want, absum, d, dtype, ("strided", dtype, pad))
    assert (wide[:, n:] == 7).all()


def MxScaled(r, e):
    return P.MxRows(r.codes, r.scales + e if e >= 0 else r.scales - (-e), r.dim)


def test_scores_nan_blocks_reach_their_rows_alone():
    dev = device()
    nq, n, d = 20, 70, 200
    q, qv = make(3, nq, d, 4, dev)
    r, rv = make(4, n, d, 4, dev)
    q.scales[7, 6] = 255   # the last, padded block
    r.scales[33, 0] = 255
    r.scales[69, 6] = 255
    got = P.mx_scores(q, r)
    bad = torch.zeros((nq, n), dtype=torch.bool)
    bad[7] = True
    bad[:, 33] = True
    bad[:, 69] = True
    assert torch.equal(torch.isnan(got).cpu(), bad)
    keep = ~bad.numpy()
    want, absum = mx.scores(qv, rv), np.abs(qv) @ np.abs(rv).T
    assert (np.abs(f64(got) - want)[keep] <= (2 * (d + 16) * 2.0 ** -24 * absum)[keep]).all()


def test_scores_extreme_scales():
    """Scales at the format's ends: products under- and overflow as their values do."""
    dev = device()
    q, qv = make(8, 3, 64, 4, dev)
    r, rv = make(9, 20, 64, 4, dev)
    q.scales[:] = torch.tensor([[0, 1], [254, 254], [127, 127]], dtype=torch.uint8)
    r.scales[:10], r.scales[10:] = 254, 127
    got = f64(P.mx_scores(q, r))
    qv = mx.values(*stored(q), 64, 4)
    rv = mx.values(*stored(r), 64, 4)
    want = mx.scores(qv, rv)
    assert (np.abs(got[0, :10] - want[0, :10]) <= 2 * 80 * 2.0 ** -24 * (np.abs(qv[:1]) @ np.abs(rv[:10]).T)[0] + 1e-38).all()
    assert (np.abs(got[2, 10:] - want[2, 10:]) <= 2 * 80 * 2.0 ** -24 * (np.abs(qv[2:]) @ np.abs(rv[10:]).T)[0]).all()
    assert (np.abs(want[2, :10]) > 2.0 ** 128).all() and not np.isfinite(got[1:, :10]).any()  # past fp32


def test_scores_offsets_past_32_bits():
    dev = device()
    nq, n, d = 70001, 32771, 64  # 2.3e9 scores
    q, qv = make(21, nq, d, 4, dev)
    r, rv = make(22, n, d, 4, dev)
    log("scores", nq, n, d)
    s = P.mx_scores(q, r, torch.bfloat16)
    iq = np.array([0, 1, 32767, 65534, 65535, 65536, 70000])
    want, absum = mx.scores(qv[iq], rv), np.abs(qv[iq]) @ np.abs(rv).T
    check_sums(s[torch.from_numpy(iq).to(dev)], want, absum, d, "bf16", "long")


def test_scores_of_none():
    dev = device()
    a, b = P.MxRows.empty(0, 64), P.mx_quantize(draw(1, 5, 64).to(dev))
    assert P.mx_scores(a, b).shape == (0, 5) and P.mx_scores(b, a).shape == (5, 0)
    assert len(P.mx_quantize(torch.empty((0, 64), device=dev))) == 0 and P.mx_values(a).shape == (0, 64)
    g = P.mx_scores_grad(torch.empty((5, 0), device=dev), a)
    assert g.shape == (5, 64) and not g.any()
    g = P.mx_scores_grad(torch.empty((0, 3), device=dev), a, transposed=True)
    assert g.shape == (3, 64) and not g.any()
    assert P.mx_scores_grad(torch.empty((0, 5), device=dev), b).shape == (0, 64)


# ------------------------------------------------------------------------------------- the products' gradient
GRADS = [(1, 1, 1), (1, 5, 33), (3, 64, 32), (16, 100, 128), (17, 33, 100), (1, 5000, 384), (64, 1000, 256), (100, 77, 1024),
         (129, 300, 160), (257, 129, 96), (5, 31, 8192), (40, 3000, 768), (300, 513, 416), (2, 20001, 130), (1000, 65, 200)]


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("m,k,d", GRADS)
def test_scores_grad_matches_the_oracle(bits, dtype, transposed, m, k, d):
    dev = device()
    log("grad", bits, dtype, transposed, m, k, d)
    x, xv = make(m + d, k, d, bits, dev)
    g = np.random.default_rng(m * 7 + k)
    gv = g.normal(size=(k, m) if transposed else (m, k)) * 2.0 ** g.integers(-12, 4, size=(k, m) if transposed else (m, k))
    gt = torch.from_numpy(gv).to(DT[dtype])
    gv = f64(gt)
    want = mx.scores_grad(gv, xv, transposed)
    absum = mx.scores_grad(np.abs(gv), np.abs(xv), transposed)
    got = P.mx_scores_grad(gt.to(dev), x, transposed)
    assert got.dtype == torch.float32
    check_sums(got, want, absum, k, "f32", (bits, dtype, transposed, m, k, d))
    again = P.mx_scores_grad(gt.to(dev), x, transposed)
    assert torch.equal(got, again)  # a fixed order


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("pad", [1, 2, 3, 8])
def test_scores_grad_of_strided_gradients(dtype, transposed, pad):
    dev = device()
    m, k, d = 45, 210, 100
    x, xv = make(6, k + 11, d, 4, dev)
    shape = (k, m) if transposed else (m, k)
    wide = draw(7, shape[0], shape[1] + pad, dtype, unit=False).to(dev)
    out = torch.full((m, d + pad), 7.0, device=dev)
    P.mx_scores_grad(wide[:, :shape[1]], x.part(11, k), transposed, out=out[:, :d])
    gv = f64(wide[:, :shape[1]])
    check_sums(out[:, :d], mx.scores_grad(gv, xv[11:], transposed), mx.scores_grad(np.abs(gv), np.abs(xv[11:]), transposed), k,
               "f32", (dtype, transposed, pad))
    assert (out[:, d:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_scores_grad_nan_and_infinity(dtype, transposed):
    """NaN blocks, and NaN or infinite gradients, reach the outputs that their terms belong to and no other; what lies
    past the rows and columns meant is not read into them."""
    dev = device()
    m, k, d = 21, 50, 96
    x, xv = make(8, k + 3, d, 4, dev)
    x.scales[k:] = 255
    x.scales[9, 1] = 255                       # elements 32 .. 63 of row 9
    shape = (k, m) if transposed else (m, k)
    wide = torch.full((shape[0] + 1, shape[1] + 5), float("nan"), dtype=DT[dtype], device=dev)
    wide[:shape[0], :shape[1]] = draw(9, *shape, dtype, unit=False).to(dev)
    g = wide[:shape[0], :shape[1]]
    at = lambda i, j: (j, i) if transposed else (i, j)
    g[at(4, 7)] = float("inf")
    g[at(6, 3)] = float("nan")
    got = f64(P.mx_scores_grad(g, x.part(0, k), transposed))
    fine = np.ones((m, d), dtype=bool)
    fine[:, 32:64] = False
    assert np.isnan(got[:, 32:64]).all()
    row4 = got[4, np.r_[0:32, 64:96]]
    term = xv[7, np.r_[0:32, 64:96]]
    assert (np.isnan(row4) | (np.isinf(row4) & (np.sign(row4) == np.sign(term)))).all() and not np.isfinite(row4).any()
    assert np.isnan(got[6]).all()
    fine[[4, 6]] = False
    gv = f64(g).T if transposed else f64(g)
    gv = np.where(np.isfinite(gv), gv, 0)
    tol = 2 * (k + 16) * 2.0 ** -24 * (np.abs(gv) @ np.abs(xv[:k]))
    assert (np.abs(got - gv @ xv[:k])[fine] <= tol[fine]).all()


def test_scores_grad_keeps_small_gradients_of_fp32():
    """Gradients far below a row's largest still count in full: sums of them alone are as exact as any."""
    dev = device()
    m, k, d = 8, 64, 64
    x, xv = make(12, k, d, 4, dev)
    g = np.random.default_rng(1).normal(size=(m, k)).astype(np.float32)
    g[:, 0] = 2.0 ** 60
    x.codes[0] = 0
    g[4:] *= 2.0 ** -90
    g[4:, 0] = 1.0
    xv[0] = 0
    got = P.mx_scores_grad(torch.from_numpy(g).to(dev), x)
    gv = g.astype(np.float64)
    gv[:, 0] = 0
    check_sums(got, gv @ xv, np.abs(gv) @ np.abs(xv), k, "f32", "small")


@pytest.mark.parametrize("transposed", [False, True])
def test_scores_grad_offsets_past_32_bits(transposed):
    dev = device()
    m, k, d = (3, 40, 64) if not transposed else (40, 3, 64)
    ld = (1 << 30) + 64
    buf = torch.empty(3 * ld, dtype=torch.bfloat16, device=dev)
    g = buf.as_strided((3, 40), (ld, 1))
    g.copy_(draw(13, 3, 40, "bf16", unit=False))
    x, xv = make(14, k, d, 6, dev)
    gv = f64(g)
    got = P.mx_scores_grad(g, x, transposed)
    check_sums(got, mx.scores_grad(gv, xv, transposed), mx.scores_grad(np.abs(gv), np.abs(xv), transposed), k, "f32", "far")


def test_scores_grad_is_the_scores_derivative():
    """Differences of the products themselves: S is linear in the values, so whole steps are exact up to rounding."""
    dev = device()
    nq, n, d = 6, 40, 64
    q, qv = make(15, nq, d, 4, dev)
    r, rv = make(16, n, d, 4, dev)
    up = draw(17, nq, n, unit=False)
    dq = f64(P.mx_scores_grad(up.to(dev), r))
    codes, scales = stored(q)
    base = (f64(up) * f64(P.mx_scores(q, r))).sum()
    for i, j in ((0, 0), (2, 33), (5, 63)):
        c2 = codes.copy()
        c2[i, j // 32, j % 32] ^= 8                    # the element's sign turned
        q2 = P.MxRows(torch.from_numpy(mx.pack(c2, 4)).to(dev), q.scales, d)
        step = (f64(up) * f64(P.mx_scores(q2, r))).sum() - base
        tol = 4 * 80 * 2.0 ** -24 * (np.abs(f64(up)) * (np.abs(qv) @ np.abs(rv).T)).sum()
        assert abs(step - dq[i, j] * -2 * qv[i, j]) <= tol


# ------------------------------------------------------------------------------------- streams, graphs, workspaces
def test_calls_run_on_the_current_stream_and_replay_in_a_graph():
    dev = device()
    nq, n, d = 48, 3000, 256
    x0, rows0 = draw(31, nq, d).to(dev), draw(32, n, d, "bf16").to(dev)
    up0 = draw(33, nq, n, unit=False).to(dev)

    def work(x, rows, up):
        q, r = P.mx_quantize(x, 6), P.mx_quantize(rows, 4)
        return P.mx_scores(q, r), P.mx_scores_grad(up, r), P.mx_scores_grad(up, q, transposed=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = work(x0, rows0, up0)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(on_side, work(x0, rows0, up0)):
        assert torch.equal(a, b)
    xs, rs, us = x0.clone(), rows0.clone(), up0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work(xs, rs, us)
    for i in range(4):
        xs.copy_(x0.roll(i, 0))
        rs.copy_(rows0.roll(3 * i, 0))
        us.copy_(up0 * (i + 1))
        want = work(xs, rs, us)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_grad_does_not_depend_on_its_workspace():
    dev = device()
    m, k, d = 20, 9000, 384
    x, _ = make(41, k, d, 4, dev)
    g = draw(42, m, k, unit=False).to(dev)
    want = P.mx_scores_grad(g, x)
    need = ctypes.c_size_t()
    desc = x._desc()
    lib = P.library()
    assert lib.oprag_mx_scores_grad_bytes(m, desc, ctypes.byref(need)) == 0
    for fill in (0, 0xFF):
        ws = torch.full((need.value + 256,), fill, dtype=torch.uint8, device=dev)
        out = torch.full((m, d), 7.0, device=dev)
        assert lib.oprag_mx_scores_grad(g.data_ptr(), 0, k, 0, m, desc, out.data_ptr(), d, ws.data_ptr(), need.value,
                                        torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(out, want) and (ws[need.value:] == fill).all()
