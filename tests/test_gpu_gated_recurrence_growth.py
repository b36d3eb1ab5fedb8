"""Gated recurrence with exponential gates above 0: products of decays that pass what fp32 holds, while the states
and gradients themselves do not.  Bounds: those of test_gpu_gated_recurrence.py, carried along in 64 bits (their terms are
relative to sizes that grow with the values; the decay of four rows or more, a rounded sum of gates and its exponential, costs
10 u and (|z| + 1) u a row, where the bound has 8 u and (|z| + 4) u a row)."""
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_gated_recurrence import _built, check, normal  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = [(8, "f32"), (5, "bf16"), (72, "bf16")]


@pytest.mark.parametrize("f,dt", WIDTHS)
@pytest.mark.parametrize("n,z", [(256, 1.0), (130, 80.0), (4500, 0.03125), (9000, 0.25)])
def test_a_state_of_zeros_stays(n, z, f, dt):
    """No input, no initial state; no loss but in the first row: zeros, and nothing else, whatever the gates' product."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    gate, x = torch.full((n, f), z, device="cuda", dtype=t), torch.zeros(n, f, device="cuda", dtype=t)
    off = torch.tensor([0, n], device="cuda")
    r = tfg.tfg_gated_recurrence(gate, x, off, "exp")
    assert bool((r.out == 0).all()) and bool((r.final == 0).all()) and bool((r.checkpoints == 0).all())
    g = torch.zeros(n, f, device="cuda", dtype=t)
    g[0] = 1.0
    b = tfg.tfg_gated_recurrence_backward(gate, x, off, r.checkpoints, g, "exp", initial=torch.zeros(1, f, device="cuda"))
    assert bool((b.x[1:] == 0).all()) and torch.equal(b.x[:1], g[:1]) and bool((b.gate == 0).all())


@pytest.mark.parametrize("f,dt", WIDTHS)
def test_channels_of_zeros_beside_others(f, dt):
    """As a ReLU leaves them: channels without input beside channels with it, gates of both signs around 0.02."""
    n = 3000
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    gate = (0.02 + 0.2 * torch.randn(n, f, device="cuda", generator=gen)).to(t)
    x = torch.randn(n, f, device="cuda", generator=gen).to(t)
    x[:, ::2] = 0
    x[2800:, ::2] = 1
    g = normal(n, f, 5, dt) * 1e-20
    r, _ = check(gate, x, [0, n], "exp", None, "f32", g.float(), None)
    assert bool((r.out[:2800, ::2] == 0).all())


@pytest.mark.parametrize("f,dt", WIDTHS)
@pytest.mark.parametrize("start,last,blocks", [
    (1e-30, 1e-5, [(100, 1.0), (100, -1.0), (130, 1.0), (120, -1.0), (20, 3.0)]),
    (1e30, 1e-30, [(128, -1.0), (128, 1.0), (8, -12.5), (8, 12.5), (300, -0.5), (270, 0.5)]),
    (1e-30, 1e-35, [(5000, 0.029052734375)]),                      # a window and more: e^145
    (1e-30, 1e20, [(16, 8.0), (16, -8.0)] * 20),
    (1.0, 1e5, [(2, 30.0), (2, -30.0)] * 2 + [(1, 80.0), (1, -80.0)] * 80)])
def test_states_that_come_back(start, last, blocks, f, dt):
    """States far from 1, cut down or raised by more than fp32 has and back.  No value on the way leaves fp32: the states
    are start e^(sum of the gates so far), the adjoint is last e^(sum of the gates still to come)."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    below = torch.cumsum(torch.tensor([0.0] + [rows * z for rows, z in blocks], dtype=torch.float64), 0)
    sizes = torch.cat([start * torch.exp(below), last * torch.exp(below[-1] - below)])
    assert 1e-37 < float(sizes.min()) and float(sizes.max()) < 1e37
    gate = torch.cat([torch.full((rows, f), z) for rows, z in blocks]).cuda().to(t)
    n = gate.shape[0]
    signs = torch.tensor([1.0, -1.5, 1.25, -1.0]).repeat(f // 4 + 1)[:f].cuda()
    initial = (start * signs)[None].contiguous()
    x = torch.zeros(n, f, device="cuda", dtype=t)
    g = torch.zeros(n, f, device="cuda")
    g[-1] = last
    check(gate, x, [0, n], "exp", initial, "f32", g, None)


def test_gates_that_forget_among_gates_that_grow():
    n, f = 700, 8
    gate = torch.full((n, f), 0.75, device="cuda")
    gate[100::100] = -float("inf")
    x = torch.zeros(n, f, device="cuda")
    x[100::100] = normal(6, f, 1) * 1e-20
    g = normal(n, f, 2) * 1e-20
    r, _ = check(gate, x, [0, n], "exp", normal(1, f, 3) * 1e-20, "f32", g, None)
    assert torch.equal(r.out[300], x[300])
