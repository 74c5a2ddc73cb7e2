"""The products' gradient at sizes that fill the GPU with large tiles, against the fp64 oracle (bounds as in
test_gpu_mx.py: sums of K fp32 terms)."""
import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import mx
from tests.gpu_helpers import DT, device, log
from tests.test_gpu_mx import check_sums, f64, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 6])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,k,d,pad", [(33001, 515, 40, 0), (32769, 512, 257, 3), (65536, 576, 33, 8), (17000, 1025, 600, 1)])
def test_scores_grad_of_many_rows(bits, transposed, dtype, m, k, d, pad):
    """From one round of tiles to several, the last tile short by any number of rows; strided gradients."""
    log("grad rows", bits, transposed, dtype, m, k, d, pad)
    dev = device()
    x, xv = make(m + d, k, d, bits, dev)
    g = torch.Generator().manual_seed(m)
    shape = (k, m + pad) if transposed else (m, k + pad)
    G = torch.randn(shape, generator=g).to(DT[dtype])
    G = G[:, :m] if transposed else G[:, :k]
    out = torch.full((m + 1, d + 2), 7.0, device=dev)
    on_dev = torch.empty(shape, dtype=DT[dtype], device=dev)[:, :G.shape[1]].copy_(G)
    got = P.mx_scores_grad(on_dev, x, transposed=transposed, out=out[:m, :d])
    gv = f64(G)
    want = mx.scores_grad(gv, xv, transposed)
    absum = mx.scores_grad(np.abs(gv), np.abs(xv), transposed)
    check_sums(got, want, absum, k, "f32", (bits, transposed, dtype, m, k, d))
    assert (out[m] == 7.0).all() and (out[:, d:] == 7.0).all()
