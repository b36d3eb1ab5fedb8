"""Distillation of logits and gradients that reach their 16-byte boundaries at different places, as a slice of a batch and the
gradient that the binding makes do.  Bounds: those of test_gpu_distillation.py."""
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_distillation import DT, Plain, _built, close, make  # noqa: F401

pytestmark = pytest.mark.gpu
# rows by parts of a warp (many), a warp, and CTAs of 128, 256 and 512 threads that hold a row; rows that none holds
SIZES = [(10_001, 41), (10_001, 127), (19, 41), (7, 1031), (7, 2047), (5, 4999), (4, 12_001), (4, 40_001), (3, 60_001), (3, 120_001)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", SIZES)
def test_a_slice_has_the_same_bits_with_its_gradient(n, v, dt):
    cut = 3
    logits, ids, teacher = make(n + cut, v, 7, v, dt)
    w = torch.ones(n + cut, device="cuda")
    w[cut + 1::3] = 0.0
    teacher[cut + 2] = -float("inf")
    part, ids, teacher, w = logits[cut:], ids[cut:], teacher[cut:], w[cut:]
    assert part.data_ptr() % 16 != 0
    a = dict(row_weight=w, padding_id=-1)
    alone = tfg.tfg_distillation_loss(part, ids, teacher, 1.5, **a, want_stats=True)
    # gradients at every place that a value may begin: on the logits' boundaries and off them
    step, want = logits.element_size(), None
    up = torch.linspace(-1, 2, n, device="cuda")
    p = Plain(part, ids, teacher, 1.5, w)
    for first in range(0, 16 // step + 1, 1 if n < 1000 else 3):
        room = torch.full((n * v + 40,), 5.0, dtype=DT[dt], device="cuda")
        grad = room[16 + first:16 + first + n * v].view(n, v)
        both = tfg.tfg_distillation_loss(part, ids, teacher, 1.5, **a, want_stats=True, grad_logits=grad)
        assert torch.equal(both.loss, alone.loss) and torch.equal(both.stats, alone.stats)
        if want is None:
            close(both.loss, p.loss, p.loss_tol, "loss")
            close(grad, *p.grad(), "gradient")
            want = grad.clone()
        assert torch.equal(grad, want), "the gradient's bits do not hang on where it lies"
        assert bool((room[:16 + first] == 5).all()) and bool((room[16 + first + n * v:] == 5).all())
        room.fill_(5.0)
        tfg.tfg_distillation_loss_backward(part, ids, teacher, 1.5, alone.stats, up, grad_logits=grad, **a)
        if first == 0:
            close(grad, *p.grad(up), "backward")
            back = grad.clone()
        assert torch.equal(grad, back)
        assert bool((room[:16 + first] == 5).all()) and bool((room[16 + first + n * v:] == 5).all())


def test_rows_that_count_for_nothing():
    """Weight 0, or no teacher entry above -inf: zeros whatever the logits hold, and statistics of (0, 1)."""
    for v in (41, 5000, 60_001):
        logits = torch.randn(8, v, device="cuda")
        logits[1], logits[2, 5], logits[3] = float("nan"), float("inf"), -float("inf")
        ids = torch.arange(8 * 4, device="cuda").view(8, 4) % v
        teacher, w = torch.zeros(8, 4, device="cuda"), torch.ones(8, device="cuda")
        w[1] = w[3] = 0.0
        teacher[2] = -float("inf")
        r = tfg.tfg_distillation_loss(logits, ids, teacher, row_weight=w, want_stats=True, want_grad=True)
        back = tfg.tfg_distillation_loss_backward(logits, ids, teacher, 1.0, r.stats, torch.ones(8, device="cuda"), row_weight=w)
        for i in (1, 2, 3):
            assert float(r.loss[i]) == 0 and r.stats[i].tolist() == [0, 1]
            assert bool((r.grad_logits[i] == 0).all()) and bool((back[i] == 0).all())
        assert bool(torch.isfinite(r.loss).all()) and bool(torch.isfinite(r.grad_logits).all())
