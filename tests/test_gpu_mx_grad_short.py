"""The rows' gradient from few queries (one or two stages of the sum, or part of one), against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import mx
from tests.gpu_helpers import DT, device, log
from tests.test_gpu_mx import check_sums, f64, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("k", [1, 5, 63, 64, 65, 100, 127, 128, 129])
@pytest.mark.parametrize("m,d", [(16, 40), (70, 288), (1000, 33), (40001, 130)])
def test_rows_gradient_from_few_queries(bits, dtype, k, m, d):
    log("rows' gradient", bits, dtype, k, m, d)
    dev = device()
    x, xv = make(m + k, k, d, bits, dev)
    G = torch.randn((k, m), generator=torch.Generator().manual_seed(k)).to(DT[dtype])
    gv = f64(G)
    got = P.mx_scores_grad(G.to(dev), x, transposed=True)
    check_sums(got, mx.scores_grad(gv, xv, True), mx.scores_grad(np.abs(gv), np.abs(xv), True), k, "f32", (bits, dtype, k, m, d))


@pytest.mark.parametrize("k", [3, 64, 70, 128])
def test_an_infinity_reaches_its_own_row_alone(k):
    """The last query's G is infinite in one place: elements beside it stay as they are (nothing past the last query is
    multiplied)."""
    dev = device()
    m, d = 300, 96
    x, xv = make(k, k, d, 4, dev)
    G = torch.randn((k, m), generator=torch.Generator().manual_seed(1))
    clean = P.mx_scores_grad(G.to(dev), x, transposed=True)
    G[k - 1, 17] = float("inf")
    got = P.mx_scores_grad(G.to(dev), x, transposed=True)
    others = [i for i in range(m) if i != 17]
    assert torch.equal(got[others], clean[others])
    row = f64(got)[17]
    np.testing.assert_array_equal(np.isnan(row), xv[k - 1] == 0)
    np.testing.assert_array_equal(row[xv[k - 1] != 0], np.sign(xv[k - 1][xv[k - 1] != 0]) * np.inf)
