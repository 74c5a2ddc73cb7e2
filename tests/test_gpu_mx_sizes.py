"""Rows in few bits at sizes that fill the GPU: the tilings taken there, passes of a grid over more blocks than it has
threads for, the shortest dimensions.  Against the fp64 oracle, with the bounds of the smaller sizes' tests."""
import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import mx
from tests.gpu_helpers import DT, device, log
from tests.test_gpu_mx import check_sums, draw, f64, make, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [2, 5, 7, 8, 9, 12, 15, 39, 63, 65])
def test_quantize_and_values_of_short_dimensions(bits, dtype, d):
    dev = device()
    log("quantize", bits, dtype, d)
    x = draw(d, 1031, d + 3, dtype)[:, :d]  # rows that begin at any element
    r = P.mx_quantize(x.to(dev), bits)
    want_c, want_s = mx.quantize(f64(x), bits)
    c, s = stored(r)
    np.testing.assert_array_equal(s, want_s)
    np.testing.assert_array_equal(c, want_c)
    want = mx.values(want_c, want_s, d, bits)
    for out in ("f32", "bf16", "f16"):
        full = torch.full((1031, d + 5), 7.0, dtype=DT[out], device=dev)
        P.mx_values(r, DT[out], out=full[:, :d])
        np.testing.assert_array_equal(f64(full[:, :d]), f64(torch.from_numpy(want).to(DT[out])))
        assert (full[:, d:] == 7).all()


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype,d", [("f32", 5), ("bf16", 40), ("f16", 129), ("bf16", 1)])
def test_quantize_and_values_of_more_blocks_than_a_grid_has(bits, dtype, d):
    dev = device()
    log("quantize", bits, dtype, d)
    base = draw(d, 1009, d, dtype, unit=False)
    n = 9_000_011 // ((d + 31) // 32)
    pick = torch.randint(0, 1009, (n,), generator=torch.Generator(dev).manual_seed(1), device=dev)
    small = P.mx_quantize(base.to(dev), bits)
    c, s = stored(small)
    want_c, want_s = mx.quantize(f64(base), bits)
    np.testing.assert_array_equal(s, want_s)
    np.testing.assert_array_equal(c, want_c)
    r = P.mx_quantize(base.to(dev)[pick], bits)
    assert torch.equal(r.scales, small.scales[pick])
    assert torch.equal(r.codes, small.codes[pick])
    values = P.mx_values(small, DT[dtype])
    assert torch.equal(P.mx_values(r, DT[dtype]), values[pick])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("qb,rb", [(4, 4), (6, 4), (4, 6), (6, 6)])
@pytest.mark.parametrize("nq,n,d", [(1025, 16901, 96), (1024, 32768, 64), (130, 65999, 160), (33, 131075, 64), (64, 140001, 33),
                                    (300, 25000, 1024), (20, 133333, 2048)])
def test_scores_of_many_rows(qb, rb, nq, n, d, dtype):
    dev = device()
    log("scores", qb, rb, nq, n, d, dtype)
    q, qv = make(nq + d, nq, d, qb, dev)
    small, rv = make(n + d, 1013, d, rb, dev)
    pick = np.random.default_rng(n).integers(0, 1013, size=n)
    scale = 2.0 ** -18 if dtype == "f16" else 1.0  # (below f16's largest)
    at = torch.from_numpy(pick).to(dev)
    r = P.MxRows(small.codes[at], small.scales[at] - (18 if dtype == "f16" else 0), d)
    want, absum = mx.scores(qv, rv) * scale, np.abs(qv) @ np.abs(rv).T * scale
    full = torch.full((nq, n + 3), 7.0, dtype=DT[dtype], device=dev)
    P.mx_scores(q, r, DT[dtype], out=full[:, :n])
    assert (full[:, n:] == 7).all()
    # Equal rows have equal sums, wherever in the rows they lie: one of each is checked against the oracle.
    got = full[:, :n]
    first = torch.empty(1013, dtype=torch.int64, device=dev)
    first[at.flip(0)] = torch.arange(n - 1, -1, -1, device=dev)
    assert torch.equal(got, got[:, first[at]])
    have = torch.unique(at)
    cols = have.cpu().numpy()
    check_sums(got[:, first[have]], want[:, cols], absum[:, cols], d, dtype, (dtype, nq, n, d))
