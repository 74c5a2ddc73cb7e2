"""Refusals of the calls on rows in few bits and of the distillation calls: bad arguments are turned down before
the device is touched (no GPU needed: no call here reaches a kernel)."""
import ctypes
import os

import pytest
import torch

import paper_2608_08340_amd as P

E_INVALID = -1
V = ctypes.c_void_p
OK_PTR = 4096


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(P.LIB_PATH):
        pytest.skip("liboprag.so not built")
    return P.library()


def rows(n=4, dim=64, bits=4, codes=OK_PTR, scales=OK_PTR, first=0):
    return P._MxDesc(codes, scales, first, n, dim, bits)


BAD_ROWS = [
    (rows(bits=5), "bits"), (rows(bits=8), "bits"), (rows(dim=0), "dim"), (rows(dim=8193), "dim"), (rows(n=-1), "rows"),
    (rows(first=-1), "first_row"), (rows(n=2**31), "rows"), (rows(n=2**30, first=2**30), "first + rows"),
    (rows(n=2**62, first=2**62), "first + rows"), (rows(codes=None), "null codes"), (rows(scales=None), "null scales"),
    (rows(codes=4104), "misaligned codes"), (rows(scales=4097), "misaligned scales"),
]


@pytest.mark.parametrize("r,why", BAD_ROWS)
def test_bad_rows_are_refused_everywhere(lib, r, why):
    sz = ctypes.c_size_t()
    assert lib.oprag_mx_quantize(V(OK_PTR), 0, 8192, r, None) == E_INVALID, why
    assert lib.oprag_last_error()
    assert lib.oprag_mx_values(r, V(OK_PTR), 0, 8192, None) == E_INVALID, why
    assert lib.oprag_mx_scores(r, rows(), V(OK_PTR), 0, 2**31, None) == E_INVALID, why
    assert lib.oprag_mx_scores(rows(), r, V(OK_PTR), 0, 2**31, None) == E_INVALID, why
    assert lib.oprag_mx_scores_grad_bytes(3, r, ctypes.byref(sz)) == E_INVALID, why
    assert lib.oprag_mx_scores_grad(V(OK_PTR), 0, 2**31, 0, 3, r, V(OK_PTR), 8192, V(OK_PTR), 1 << 40, None) == E_INVALID


def test_null_rows(lib):
    sz = ctypes.c_size_t()
    assert lib.oprag_mx_quantize(V(OK_PTR), 0, 64, None, None) == E_INVALID
    assert lib.oprag_mx_values(None, V(OK_PTR), 0, 64, None) == E_INVALID
    assert lib.oprag_mx_scores(None, rows(), V(OK_PTR), 0, 64, None) == E_INVALID
    assert lib.oprag_mx_scores(rows(), None, V(OK_PTR), 0, 64, None) == E_INVALID
    assert lib.oprag_mx_scores_grad_bytes(3, None, ctypes.byref(sz)) == E_INVALID
    assert lib.oprag_mx_scores_grad_bytes(3, rows(), None) == E_INVALID
    assert lib.oprag_mx_scores_grad(V(OK_PTR), 0, 64, 0, 3, None, V(OK_PTR), 64, None, 0, None) == E_INVALID


@pytest.mark.parametrize("ptr,dtype,ld,why", [
    (None, 0, 64, "null"), (4100, 0, 64, "misaligned"), (OK_PTR, 3, 64, "dtype"), (OK_PTR, -1, 64, "dtype"),
    (OK_PTR, 1, 63, "stride below the width"), (OK_PTR, 1, 0, "stride 0"), (OK_PTR, 1, -64, "negative stride"),
    (OK_PTR, 1, 2**31 + 1, "stride too large"),
])
def test_bad_matrices_are_refused(lib, ptr, dtype, ld, why):
    p = None if ptr is None else V(ptr)
    assert lib.oprag_mx_quantize(p, dtype, ld, rows(), None) == E_INVALID, why
    assert lib.oprag_mx_values(rows(), p, dtype, ld, None) == E_INVALID, why
    assert lib.oprag_mx_scores(rows(), rows(n=64), p, dtype, ld, None) == E_INVALID, why
    assert lib.oprag_mx_scores_grad(p, dtype, ld, 0, 3, rows(n=64), V(OK_PTR), 64, V(OK_PTR), 1 << 40, None) == E_INVALID
    assert lib.oprag_mx_scores_grad(p, dtype, ld, 1, 64, rows(n=3), V(OK_PTR), 64, V(OK_PTR), 1 << 40, None) == E_INVALID
    if dtype in (0, 1):
        assert lib.oprag_mx_scores_grad(V(OK_PTR), 0, 64, 0, 3, rows(n=64), p, ld, V(OK_PTR), 1 << 40, None) == E_INVALID
    a = (ctypes.c_int64(4), ctypes.c_int64(64), V(OK_PTR), V(OK_PTR), 5, 1.0, 1.0)
    assert lib.oprag_distill_loss(p, dtype, ld, *a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 1 << 40, None) == E_INVALID, why
    assert lib.oprag_distill_grad(p, dtype, ld, *a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 64, None) == E_INVALID, why
    assert lib.oprag_distill_step(p, dtype, ld, *a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 64, V(OK_PTR), 1 << 40, None) == E_INVALID
    if dtype in (0, 1):  # the gradient's own matrix
        assert lib.oprag_distill_grad(V(OK_PTR), dtype, 64, *a, V(OK_PTR), V(OK_PTR), p, ld, None) == E_INVALID, why


def test_widths_must_agree(lib):
    assert lib.oprag_mx_scores(rows(dim=64), rows(dim=96), V(OK_PTR), 0, 64, None) == E_INVALID
    assert b"dim" in lib.oprag_last_error()


@pytest.mark.parametrize("m,tr", [(-1, 0), (2**31, 0), (3, 2), (3, -1)])
def test_grad_refuses(lib, m, tr):
    assert lib.oprag_mx_scores_grad(V(OK_PTR), 0, 2**31, tr, m, rows(), V(OK_PTR), 64, V(OK_PTR), 1 << 40, None) == E_INVALID


def test_grad_checks_its_workspace(lib):
    sz = ctypes.c_size_t()
    r = rows(n=1 << 20, dim=1024)
    assert lib.oprag_mx_scores_grad_bytes(1, r, ctypes.byref(sz)) == 0
    if sz.value:
        for ws, size in ((None, sz.value), (V(4100), sz.value), (V(OK_PTR), sz.value - 1)):
            assert lib.oprag_mx_scores_grad(V(OK_PTR), 0, 1 << 20, 0, 1, r, V(OK_PTR), 1024, ws, size, None) == E_INVALID


@pytest.mark.parametrize("nq,n,k,ids,t,tau,ttau,why", [
    (-1, 64, 5, OK_PTR, OK_PTR, 1, 1, "nq"), (2**31, 64, 5, OK_PTR, OK_PTR, 1, 1, "nq"),
    (4, -1, 5, OK_PTR, OK_PTR, 1, 1, "n"), (4, 2**31, 5, OK_PTR, OK_PTR, 1, 1, "n"),
    (4, 64, 0, OK_PTR, OK_PTR, 1, 1, "k"), (4, 64, 129, OK_PTR, OK_PTR, 1, 1, "k"),
    (4, 64, 5, None, OK_PTR, 1, 1, "null ids"), (4, 64, 5, OK_PTR, None, 1, 1, "null scores"),
    (4, 64, 5, 4104, OK_PTR, 1, 1, "misaligned ids"), (4, 64, 5, OK_PTR, 4100, 1, 1, "misaligned scores"),
    (4, 64, 5, OK_PTR, OK_PTR, 0, 1, "temperature"), (4, 64, 5, OK_PTR, OK_PTR, -1, 1, "temperature"),
    (4, 64, 5, OK_PTR, OK_PTR, float("nan"), 1, "temperature"), (4, 64, 5, OK_PTR, OK_PTR, float("inf"), 1, "temperature"),
    (4, 64, 5, OK_PTR, OK_PTR, 1e-40, 1, "temperature"),
    (4, 64, 5, OK_PTR, OK_PTR, 1, 0, "teacher temperature"), (4, 64, 5, OK_PTR, OK_PTR, 1, float("nan"), "teacher temp."),
])
def test_distill_refuses(lib, nq, n, k, ids, t, tau, ttau, why):
    p = lambda v: None if v is None else V(v)
    a = (V(OK_PTR), 0, 2**31, nq, n, p(ids), p(t), k, tau, ttau)
    assert lib.oprag_distill_loss(*a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 1 << 40, None) == E_INVALID, why
    assert lib.oprag_distill_grad(*a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 2**31, None) == E_INVALID, why
    assert lib.oprag_distill_step(*a, V(OK_PTR), V(OK_PTR), V(OK_PTR), 2**31, V(OK_PTR), 1 << 40, None) == E_INVALID, why


def test_distill_refuses_missing_outputs(lib):
    a = (V(OK_PTR), 0, 64, 4, 64, V(OK_PTR), V(OK_PTR), 5, 1.0, 1.0)
    big = (V(OK_PTR), 1 << 40, None)
    assert lib.oprag_distill_loss(*a, None, V(OK_PTR), *big) == E_INVALID
    assert lib.oprag_distill_loss(*a, V(OK_PTR), None, *big) == E_INVALID
    assert lib.oprag_distill_grad(*a, None, V(OK_PTR), V(OK_PTR), 64, None) == E_INVALID
    assert lib.oprag_distill_grad(*a, V(OK_PTR), None, V(OK_PTR), 64, None) == E_INVALID
    assert lib.oprag_distill_step(*a, None, V(OK_PTR), V(OK_PTR), 64, *big) == E_INVALID
    assert lib.oprag_distill_step(*a, V(OK_PTR), None, V(OK_PTR), 64, *big) == E_INVALID
    sz = ctypes.c_size_t()
    assert lib.oprag_distill_bytes(4, 64, None) == E_INVALID
    assert lib.oprag_distill_bytes(-4, 64, ctypes.byref(sz)) == E_INVALID
    assert lib.oprag_distill_bytes(4, 2**31, ctypes.byref(sz)) == E_INVALID


def test_nothing_to_do_is_no_error(lib):
    none = rows(n=0, codes=None, scales=None)
    assert lib.oprag_mx_quantize(None, 0, 0, none, None) == 0
    assert lib.oprag_mx_values(none, None, 0, 0, None) == 0
    assert lib.oprag_mx_scores(none, rows(), None, 0, 0, None) == 0
    assert lib.oprag_mx_scores(rows(), none, None, 0, 0, None) == 0
    assert lib.oprag_mx_scores_grad(None, 0, 0, 0, 0, rows(), None, 0, None, 0, None) == 0
    assert lib.oprag_distill_loss(None, 0, 0, 0, 64, None, None, 5, 1.0, 1.0, None, None, None, 0, None) == 0
    assert lib.oprag_distill_grad(None, 0, 0, 0, 64, None, None, 5, 1.0, 1.0, None, None, None, 0, None) == 0
    assert lib.oprag_distill_step(None, 0, 0, 0, 64, None, None, 5, 1.0, 1.0, None, None, None, 0, None, 0, None) == 0


def test_binding_refuses_what_the_library_cannot_take():
    u8 = torch.uint8
    ok = P.MxRows(torch.zeros(4, 2, 16, dtype=u8), torch.zeros(4, 2, dtype=u8), 64)
    assert len(ok) == 4 and ok.bits == 4 and len(ok.part(1, 3)) == 3 and ok.part(1, 3).part(2, 1).first == 3
    for f in (lambda: P.MxRows(torch.zeros(4, 2, 15, dtype=u8), torch.zeros(4, 2, dtype=u8), 64),
              lambda: P.MxRows(torch.zeros(4, 2, 16, dtype=u8), torch.zeros(4, 3, dtype=u8), 64),
              lambda: P.MxRows(torch.zeros(4, 2, 16, dtype=u8), torch.zeros(4, 2, dtype=u8), 65),
              lambda: P.MxRows(torch.zeros(4, 2, 16), torch.zeros(4, 2, dtype=u8), 64),
              lambda: P.MxRows(torch.zeros(4, 2, 32, dtype=u8)[:, :, ::2], torch.zeros(4, 2, dtype=u8), 64),
              lambda: ok.part(2, 3), lambda: ok.part(-1, 1), lambda: ok.part(1, 3).part(1, 3),
              lambda: P.MxRows.empty(4, 64, 5),
              lambda: P.mx_quantize(torch.zeros(4, 64)),          # not on a GPU
              lambda: P.mx_values(ok), lambda: P.mx_scores(ok, ok), lambda: P.mx_scores_grad(torch.zeros(4, 4), ok),
              lambda: P.mx_scores(torch.zeros(4, 64), ok), lambda: P.mx_quantize(torch.zeros(4)),
              lambda: P.distill_loss(torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2))):
        with pytest.raises(P.OpragError):
            f()
