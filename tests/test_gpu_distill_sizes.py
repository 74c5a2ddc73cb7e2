"""Distillation at the lengths where its launches change, against the fp64 oracle (bounds as in test_gpu_distill.py)."""
import pytest
import torch

import paper_2608_08340_amd as P
from tests.gpu_helpers import device, log
from tests.test_gpu_distill import draw, run_all

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [4095, 4096, 4097, 8191, 8192, 8193, 24575, 24576, 24577, 16383, 16384, 16385, 32767, 32768, 32769, 40961])
def test_distill_at_the_ends_of_a_row_or_piece(dtype, n):
    log("distill", dtype, n)
    run_all(*draw(n, 3, n, 20, dtype), 0.05, 0.5, dtype, (dtype, n))


def test_distill_over_more_pieces_than_one_workgroup_joins():
    log("distill 2.2M")
    run_all(*draw(22, 2, 2200003, 100, "bf16"), 0.05, 0.5, "bf16", ("2.2M",))


def test_distill_of_more_queries_than_a_launch_has():
    log("distill 32,800 queries")
    run_all(*draw(23, 32800, 5, 3, "f32"), 0.05, 0.5, "f32", ("32,800 queries",))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [300, 5000, 32768, 50000])
def test_distill_in_place_with_entries_of_no_weight(dtype, n):
    """All but a list's first entry have probabilities that round to 0: their rows' gradients are the student's."""
    dev = device()
    log("distill in place", dtype, n)
    s, ids, t, w = draw(n + 1, 4, n, 128, dtype)
    t = torch.where(torch.isfinite(t), -60.0 * torch.arange(128.0), t)
    a = (ids.to(dev), t.to(dev), w.to(dev))
    loss, grad = P.distill_step(s.to(dev), *a, 0.05, 0.5)
    buf = s.to(dev)
    loss2, grad2 = P.distill_step(buf, *a, 0.05, 0.5, out=buf)
    assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
    run_all(s, ids, t, w, 0.05, 0.5, dtype, (dtype, n))
