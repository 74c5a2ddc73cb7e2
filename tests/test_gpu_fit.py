"""Quantisation, products, distillation and the products' gradient one after the other, as an encoder is fitted: the chain
against the fp64 oracle's, and the example that fits one."""
import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import distill as od
from oracle import mx
from tests.gpu_helpers import DT, device, log
from tests.test_gpu_mx import draw, f64, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,row_bits,dtype", [(6, 4, "f32"), (4, 4, "bf16"), (6, 6, "f16")])
@pytest.mark.parametrize("nq,n,d,k", [(1, 257, 100, 1), (37, 1003, 384, 20), (130, 5001, 128, 128)])
def test_chain_matches_the_oracle(bits, row_bits, dtype, nq, n, d, k):
    """Each stage's error is carried on: a score's (sums of d terms, then the output type's rounding) moves a
    probability by a factor of at most exp(2 delta), delta the largest of a query's over the temperature; what the
    gradient's elements are off by (and their own rounding) reaches dq times the rows' magnitudes."""
    log("chain", bits, row_bits, dtype, nq, n, d, k)
    dev = device()
    tau, ttau = 0.1, 0.5
    g = np.random.default_rng(n + d)
    x, rows = draw(n, nq, d), draw(n + 1, n, d, "bf16")
    q, r = P.mx_quantize(x.to(dev), bits), P.mx_quantize(rows.to(dev), row_bits)
    ids = torch.from_numpy(np.stack([g.permutation(n)[:k] for _ in range(nq)]))
    t = torch.from_numpy(-np.sort(-g.normal(size=(nq, k)).astype(np.float32), axis=1))
    w = torch.from_numpy(g.uniform(0.5, 2, nq).astype(np.float32))
    s = P.mx_scores(q, r, DT[dtype])
    loss, ds = P.distill_step(s, ids.to(dev), t.to(dev), w.to(dev), tau, ttau, out=s)
    dq = P.mx_scores_grad(ds, r)

    qv, rv = mx.values(*stored(q), d, bits), mx.values(*stored(r), d, row_bits)
    for got, src, b in ((qv, x, bits), (rv, rows, row_bits)):
        np.testing.assert_array_equal(got, mx.values(*mx.quantize(f64(src), b), d, b))
    S = mx.scores(qv, rv)
    want_loss, _, G = od.distill(S, ids.numpy(), t.numpy(), tau, ttau, f64(w))
    want = mx.scores_grad(G, rv)

    half = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    small = {"f32": 0.0, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}[dtype]
    err_s = 2 * (d + 16) * 2.0 ** -24 * (np.abs(qv) @ np.abs(rv).T) + 1.01 * half * np.abs(S) + small
    delta = err_s.max(axis=1) / tau
    top = np.abs(S).max(axis=1) / tau
    eps = 2.0 ** -24 * (4 * top + 4 * np.log(n + 1) + 64 + n / 64)      # of a probability, the scores given
    eps_t = 2.0 ** -24 * (8 * np.abs(t.numpy()).max(axis=1) / ttau + 64 + k)
    z = S / tau
    prob = np.exp(z - z.max(axis=1, keepdims=True))
    prob /= prob.sum(axis=1, keepdims=True)
    pt = np.zeros_like(prob)
    for i in range(nq):
        for at, p, _ in od.teacher(ids[i].tolist(), t[i].tolist(), n, ttau):
            pt[i, at] += p
    # the loss: sum p (log p - z) + lse moves by at most delta twice over
    tol = 2 * delta + eps + eps_t * (1 + 2 * top + 2 * np.abs(t.numpy()).max(axis=1) / ttau + np.log(n + 1)) \
        + 2.0 ** -22 * (top + np.abs(want_loss))
    assert (np.abs(f64(loss) - want_loss) <= tol).all()
    err_g = f64(w)[:, None] / tau * (prob * (np.expm1(2 * delta) + 2 * eps)[:, None] + pt * eps_t[:, None]
                                     + 2.0 ** -22 * (prob + pt))
    err_g += 1.01 * half * (np.abs(G) + err_g) + small
    tol = err_g @ np.abs(rv) + 2 * (n + 16) * 2.0 ** -24 * ((np.abs(G) + err_g) @ np.abs(rv))
    assert (np.abs(f64(dq) - want) <= tol).all(), (np.abs(f64(dq) - want) / tol).max()


def test_example_fits_its_queries():
    """The distortion has an inverse, so the loss falls and the lists come closer to the teacher's."""
    from examples.fit_queries import fit

    (loss0, recall0), (loss1, recall1) = fit(n=4096, dim=128, batch=128, k=16, steps=40)
    log("fit", loss0, loss1, recall0, recall1)
    assert np.isfinite([loss0, loss1]).all() and loss1 < loss0 and recall1 > recall0
