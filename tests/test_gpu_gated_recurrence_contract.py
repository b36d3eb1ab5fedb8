"""What a call of the gated recurrence hands back beside its values."""
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_gated_recurrence import _built, batch, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [100, 300])
def test_the_backward_hands_its_status_back(n):
    z, x = batch(n, 8, "sigmoid", "f32", 1)
    off = torch.tensor([0, 40, n], device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, x)
    tfg.check_status(b.status)
    gate, grad_x, initial = b                                # the three gradients, as ever
    assert len(b) == 3 and initial is None and gate is b.gate and grad_x is b.x
    bad = torch.tensor([0, 40, n + 1], device="cuda")
    b = tfg.tfg_gated_recurrence_backward(z, x, bad, r.checkpoints, x)
    assert int(b.status) == tfg.TFG_ERR_INDEX_RANGE
    with pytest.raises(tfg.TfgError):
        tfg.check_status(b.status)
    mine = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, x, status=mine)
    assert b.status is mine and int(mine) == 0
