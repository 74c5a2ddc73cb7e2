"""The distillation loss and its gradient on the GPU against the fp64 oracle.

With Z the largest |z| = |logit / temperature| of a query, a probability is off by a factor of at most
1 + eps, eps = 2^-24 (4 Z + 4 log n + 64 + n / 64): the rounding of z, of the exponential's argument and of lse (absolute
errors in the exponent), the exponential itself, and sums of n terms of which no thread adds more than n / 64
one after the other."""
import math

import numpy as np
import pytest
import torch

import paper_2608_08340_amd as P
from oracle import distill as od
from tests.gpu_helpers import DT, device, log

pytestmark = pytest.mark.gpu

HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def draw(seed, nq, n, k, dtype, masked=0.0):
    """Logits, ranked lists (some short, some empty, some entries past the rows, repeated ids) and weights."""
    g = np.random.default_rng(seed)
    s = torch.from_numpy((0.3 * g.normal(size=(nq, n))).astype(np.float32))
    if masked:
        s[torch.from_numpy(g.random((nq, n)) < masked)] = -math.inf
    ids = g.integers(0, max(n, 1), size=(nq, k))
    t = -np.sort(-g.normal(size=(nq, k)).astype(np.float32), axis=1)
    for q in range(nq):
        length = k if g.random() < 0.6 else int(g.integers(0, k + 1))
        ids[q, length:] = -1
        t[q, length:] = -np.inf
        if k > 2 and g.random() < 0.3:
            ids[q, 1] = ids[q, 0]                      # twice the same row
        if g.random() < 0.2:
            ids[q, 0] = n + int(g.integers(0, 5))      # no such row
    if masked:  # the teacher keeps to rows that are there, in all but the first query
        for q in range(1, nq):
            for e in range(k):
                if 0 <= ids[q, e] < n and s[q, ids[q, e]] == -math.inf:
                    ids[q, e] = -1
    w = g.uniform(0.5, 2.0, size=nq).astype(np.float32)
    return s.to(DT[dtype]), torch.from_numpy(ids), torch.from_numpy(t), torch.from_numpy(w)


def check(s, ids, t, w, tau, ttau, dtype, loss, lse, grad, label):
    sv, wv = f64(s), f64(w)
    nq, n = sv.shape
    want_loss, want_lse, want_grad = od.distill(sv, ids.cpu().numpy(), t.cpu().numpy(), tau, ttau, wv)
    z = np.abs(np.where(np.isfinite(sv), sv, 0) / tau).max(axis=1) if n else np.zeros(nq)
    u = np.abs(np.where(np.isfinite(t.cpu().numpy()), t.cpu().numpy(), 0) / ttau).max(axis=1)
    eps = 2.0 ** -24 * (4 * z + 4 * math.log(n + 1) + 64 + n / 64)
    eps_t = 2.0 ** -24 * (8 * u + 64 + ids.shape[1])

    def close(got, want, tol, what):
        got = f64(got)
        assert got.shape == want.shape, (label, what)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=f"{label} {what}")
        inf = np.isinf(want)
        np.testing.assert_array_equal(got[inf], want[inf], err_msg=f"{label} {what}")
        fin = np.isfinite(want)
        bad = np.abs(got - np.where(fin, want, 0))[fin] > np.broadcast_to(tol, want.shape)[fin]
        assert not bad.any(), (label, what, np.abs(got - want)[fin][bad][:3], np.broadcast_to(tol, want.shape)[fin][bad][:3])

    if lse is not None:
        close(lse, want_lse, eps + 2.0 ** -23 * np.abs(want_lse), "lse")
    if loss is not None:
        close(loss, want_loss, eps + eps_t * (1 + 2 * z + 2 * u + math.log(n + 1)) + 2.0 ** -23 * (z + np.abs(want_loss)), "loss")
    if grad is not None:
        prob = np.zeros_like(want_grad)
        if n:
            top = np.where(np.isfinite(sv), sv, -np.inf).max(axis=1, keepdims=True)
            with np.errstate(invalid="ignore"):
                e = np.where(np.isfinite(sv), np.exp((sv - np.where(np.isfinite(top), top, 0)) / tau), 0)
            tot = e.sum(axis=1, keepdims=True)
            prob = e / np.where(tot > 0, tot, 1)
        pt = np.zeros_like(want_grad)
        for q in range(nq):
            for i, p, _ in od.teacher(ids[q].tolist(), t[q].tolist(), n, ttau):
                pt[q, i] += p if np.isfinite(p) else 0
        scale = np.abs(wv)[:, None] / tau
        tol = scale * (prob * (2 * eps[:, None]) + pt * eps_t[:, None] + 2.0 ** -22 * (prob + pt))
        close(grad, want_grad, tol + HALF_ULP[dtype] * 1.01 * np.abs(np.where(np.isfinite(want_grad), want_grad, 0)) + SMALLEST[dtype], "grad")


def run_all(s, ids, t, w, tau, ttau, dtype, label):
    dev = device()
    a = (s.to(dev), ids.to(dev), t.to(dev))
    loss, lse = P.distill_loss(*a, tau, ttau)
    grad = P.distill_grad(*a, lse, w.to(dev), tau, ttau)
    check(s, ids, t, w, tau, ttau, dtype, loss, lse, grad, label + ("pair",))
    loss2, grad2 = P.distill_step(*a, w.to(dev), tau, ttau)
    check(s, ids, t, w, tau, ttau, dtype, loss2, None, grad2, label + ("step",))
    again = P.distill_step(*a, w.to(dev), tau, ttau)
    assert torch.equal(torch.nan_to_num(again[0]), torch.nan_to_num(loss2))
    assert torch.equal(torch.nan_to_num(again[1]), torch.nan_to_num(grad2))
    return loss2, grad2


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nq,n,k", [(1, 1, 1), (3, 2, 5), (2, 7, 3), (5, 63, 16), (4, 64, 128), (3, 65, 7), (2, 255, 100),
                                    (9, 1000, 10), (2, 1025, 64), (3, 4096, 128), (1, 8191, 100), (700, 130, 20),
                                    (2, 40000, 100), (1, 70001, 16), (300, 2050, 5)])
def test_distill_matches_the_oracle(dtype, nq, n, k):
    log("distill", dtype, nq, n, k)
    run_all(*draw(nq * 1000 + n, nq, n, k, dtype), 0.05, 0.5, dtype, (dtype, nq, n, k))


@pytest.mark.parametrize("nq,n", [(1, 300000), (3, 131072), (2, 1000003)])
def test_distill_over_long_rows(nq, n):
    for dtype in ("f32", "bf16"):
        log("distill long", dtype, nq, n)
        run_all(*draw(n, nq, n, 100, dtype), 0.07, 0.3, dtype, (dtype, nq, n))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [40, 3000, 90001])
def test_distill_with_masked_rows(dtype, n):
    s, ids, t, w = draw(77 + n, 6, n, 12, dtype, masked=0.3)
    s[3] = -math.inf                                   # nothing left
    ids[4] = -1                                        # no teacher
    s[5, :-1], s[5, -1] = -math.inf, 0.25              # one row left
    ids[5] = -1
    ids[5, 0], t[5, 0] = n - 1, 0.5
    loss, grad = run_all(s, ids, t, w, 0.1, 0.4, dtype, (dtype, n, "masked"))
    assert loss[4] == 0 and not grad[4].any() and loss[5] == 0
    lowest = torch.finfo(DT[dtype]).min                # masks of the type's lowest value act as -inf does
    low = s.clone()
    low[:3][low[:3] == -math.inf] = lowest
    if dtype != "f16":                                 # fp16's lowest is a mere -65504 / temperature: still no probability
        low = low.clamp(min=-1e30)
    dev = device()
    a, b = (P.distill_step(v[1:3].to(dev), ids[1:3].to(dev), t[1:3].to(dev), w[1:3].to(dev), 0.1, 0.4) for v in (s, low))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [50, 5000, 100000])
def test_distill_nan_and_infinity(dtype, n):
    s, ids, t, w = draw(99, 6, n, 8, dtype)
    ids[:] = torch.arange(8)
    t[:] = torch.linspace(1, 0, 8)
    s[0, n - 1] = math.nan
    s[1, n // 2] = math.inf
    s[2, 3] = math.nan                                 # in the teacher's list
    t[3, 0] = math.inf
    t[4, 0] = math.nan                                 # no entry
    s[5, 0] = math.nan
    ids[5] = -1                                        # no entries: no result to spoil
    loss, grad = run_all(s, ids, t, w, 0.1, 0.4, dtype, (dtype, n, "nan"))
    assert loss[5] == 0 and not grad[5].any() and torch.isfinite(grad[4]).all()


def test_distill_large_logits_do_not_overflow():
    s, ids, t, w = draw(5, 4, 600, 10, "f32")
    s *= 1e4
    ids[2, 0], s[2, 17] = 17, 3.0e38
    t[1] *= 1e5
    loss, grad = run_all(s[:2], ids[:2], t[:2], w[:2], 0.5, 0.5, "f32", ("large",))
    dev = device()
    loss, grad = P.distill_step(s[2:3].to(dev), torch.full((1, 1), 17, device=dev), torch.ones((1, 1), device=dev), w[2:3].to(dev))
    assert loss[0] == 0 and not grad.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,pad", [(100, 1), (100, 4), (1001, 7), (2048, 8), (70000, 3)])
def test_distill_of_strided_logits(dtype, n, pad):
    dev = device()
    s, ids, t, w = draw(n + pad, 5, n, 9, dtype)
    wide = torch.full((5, n + pad), 1000.0, dtype=DT[dtype], device=dev)
    wide[:, :n] = s.to(dev)
    out = torch.full((5, n + pad + 1), 7.0, dtype=DT[dtype], device=dev)
    want = P.distill_step(s.to(dev), ids.to(dev), t.to(dev), w.to(dev), 0.2, 0.3)
    loss, grad = P.distill_step(wide[:, :n], ids.to(dev), t.to(dev), w.to(dev), 0.2, 0.3, out=out[:, :n])
    check(s, ids, t, w, 0.2, 0.3, dtype, loss, None, grad, (dtype, n, pad))
    assert (out[:, n:] == 7).all() and (wide[:, n:] == 1000).all() and want[1].shape == grad.shape
    loss, lse = P.distill_loss(wide[:, :n], ids.to(dev), t.to(dev), 0.2, 0.3)
    grad = P.distill_grad(wide[:, :n], ids.to(dev), t.to(dev), lse, w.to(dev), 0.2, 0.3, out=out[:, :n])
    check(s, ids, t, w, 0.2, 0.3, dtype, loss, lse, grad, (dtype, n, pad))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,n", [(3, 500), (2, 40001), (1, 500000)])
def test_distill_in_place(dtype, nq, n):
    dev = device()
    s, ids, t, w = draw(n, nq, n, 30, dtype)
    a = (ids.to(dev), t.to(dev))
    loss, grad = P.distill_step(s.to(dev), *a, w.to(dev), 0.05, 0.5)
    buf = s.to(dev)
    loss2, grad2 = P.distill_step(buf, *a, w.to(dev), 0.05, 0.5, out=buf)
    assert grad2.data_ptr() == buf.data_ptr() and torch.equal(loss, loss2) and torch.equal(grad, grad2)
    buf = s.to(dev)
    lse = P.distill_loss(buf, *a, 0.05, 0.5)[1]
    want = P.distill_grad(buf, *a, lse, w.to(dev), 0.05, 0.5)
    assert torch.equal(P.distill_grad(buf, *a, lse, w.to(dev), 0.05, 0.5, out=buf), want)


def test_distill_offsets_past_32_bits():
    dev = device()
    nq, n = 5, 600
    ld = (1 << 29) + 8
    s, ids, t, w = draw(3, nq, n, 6, "bf16")
    buf = torch.empty(4 * ld + n, dtype=torch.bfloat16, device=dev).as_strided((nq, n), (ld, 1))
    buf.copy_(s)
    loss, grad = P.distill_step(buf, ids.to(dev), t.to(dev), w.to(dev), 0.1, 0.1, out=buf)
    check(s, ids, t, w, 0.1, 0.1, "bf16", loss, None, grad, ("far",))


def test_distill_of_nothing():
    dev = device()
    i64 = lambda *shape: torch.full(shape, -1, dtype=torch.int64, device=dev)
    f = lambda *shape: torch.zeros(shape, device=dev)
    loss, grad = P.distill_step(f(0, 10), i64(0, 3), f(0, 3), f(0))
    assert loss.shape == (0,) and grad.shape == (0, 10)
    loss, grad = P.distill_step(f(4, 0), i64(4, 3), f(4, 3), f(4))
    assert not loss.any() and grad.shape == (4, 0)
    loss, lse = P.distill_loss(f(4, 0), i64(4, 3), f(4, 3))
    assert not loss.any() and (lse == -math.inf).all()


def test_distill_gradient_against_differences_of_the_loss():
    dev = device()
    s, ids, t, w = draw(8, 6, 200, 10, "f32")
    tau, ttau = 0.5, 0.7
    loss, grad = P.distill_step(s.to(dev), ids.to(dev), t.to(dev), w.to(dev), tau, ttau)
    g = np.random.default_rng(0)
    way = g.normal(size=s.shape)
    at = lambda e: od.distill(f64(s) + e * way, ids.numpy(), t.numpy(), tau, ttau)[0]
    slope = f64(w) * (at(1e-5) - at(-1e-5)) / 2e-5
    np.testing.assert_allclose((f64(grad) * way).sum(axis=1), slope, rtol=1e-4, atol=1e-5)


def test_distill_streams_and_graphs():
    dev = device()
    for nq, n in ((64, 3000), (2, 200000)):
        s, ids, t, w = (v.to(dev) for v in draw(9, nq, n, 20, "f32"))

        def work(s):
            loss, lse = P.distill_loss(s, ids, t, 0.1, 0.2)
            return (loss, lse, P.distill_grad(s, ids, t, lse, w, 0.1, 0.2), *P.distill_step(s, ids, t, w, 0.1, 0.2))

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = work(s)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(got, work(s)):
            assert torch.equal(a, b)
        buf = s.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = work(buf)
        for i in range(4):
            buf.copy_(s * (1 + 0.1 * i))
            want = work(buf)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b), (nq, n, i)
