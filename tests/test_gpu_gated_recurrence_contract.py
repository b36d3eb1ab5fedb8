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


def poison(n, f, dtype):
    """What the allocator hands out next held NaN."""
    for k in (1, 2, 3):
        torch.full((k * n, f), float("nan"), dtype=dtype, device="cuda")


PADDED = {"one tile": ([3, 50, 90], 120), "no sequence": ([5], 60), "tail of tiles": ([0, 130, 300], 900),
          "from the middle": ([700, 701, 1000], 1037), "empty ones": ([40, 40, 40, 200, 200], 333)}


@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
@pytest.mark.parametrize("layout", PADDED)
@pytest.mark.parametrize("f,dt", [(8, "f32"), (72, "bf16"), (33, "f32"), (5, "bf16")])
def test_rows_outside_all_sequences_are_zeros_in_new_tensors(f, dt, layout, kind):
    """A padded batch: the projections' gradients are sums over all rows."""
    offsets, n = PADDED[layout]
    z, x = batch(n, f, kind, dt, 2)
    off = torch.tensor(offsets, device="cuda")
    lo, hi = offsets[0], offsets[-1]
    poison(n, f, z.dtype)
    r = tfg.tfg_gated_recurrence(z, x, off, kind)
    tfg.check_status(r.status)
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[lo:hi] = False
    assert bool((r.out[outside] == 0).all()) and bool(torch.isfinite(r.out).all())
    g = normal(n, f, 3, dt)
    poison(n, f, z.dtype)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind)
    for t in b[:2]:
        assert bool((t[outside] == 0).all()) and bool(torch.isfinite(t).all())
    # what is given keeps its rows, alone or with a new one beside it; the rows of sequences have the same bits
    mark = torch.full((n, f), 3.5, dtype=z.dtype, device="cuda")
    kept = tfg.tfg_gated_recurrence(z, x, off, kind, out=mark.clone())
    assert torch.equal(kept.out[outside], mark[outside]) and torch.equal(kept.out[lo:hi], r.out[lo:hi])
    poison(n, f, z.dtype)
    half = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, grad_gate=mark.clone())
    assert torch.equal(half.gate[outside], mark[outside]) and bool((half.x[outside] == 0).all())
    assert torch.equal(half.gate[lo:hi], b.gate[lo:hi]) and torch.equal(half.x[lo:hi], b.x[lo:hi])


def test_a_projections_gradient_over_a_padded_batch():
    n, f, k, offsets = 500, 32, 16, [0, 77, 300]
    h = normal(n, k, 1)
    w = normal(k, 2 * f, 2) * 0.2
    off = torch.tensor(offsets, device="cuda")
    z, x = (h @ w).chunk(2, dim=1)
    poison(n, 2 * f, torch.float32)
    r = tfg.tfg_gated_recurrence(z, x, off)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, torch.ones(n, f, device="cuda"))
    both = torch.cat([b.gate, b.x], 1)
    assert torch.equal(h.t() @ both, torch.cat([h[:300], torch.zeros_like(h[300:])]).t() @ both)
    assert bool(torch.isfinite(h.t() @ both).all()) and bool(torch.isfinite(r.out.t() @ both).all())


@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
@pytest.mark.parametrize("f,dt", [(40, "f32"), (72, "bf16"), (33, "f32")])
@pytest.mark.parametrize("lengths", [[50, 60, 70], [13, 3, 9], [400, 500, 30], [5000, 300, 4200]])
def test_gates_of_a_sequence_do_not_reach_another(lengths, f, dt, kind):
    """Nor do rows outside all sequences: the others' results stay bit for bit, whatever gates the middle one has
    and whatever lies before and behind."""
    lo, n = 21, 21 + sum(lengths) + 100
    offsets = [lo]
    for k in lengths:
        offsets.append(offsets[-1] + k)
    off = torch.tensor(offsets, device="cuda")
    z, x = batch(n, f, kind, dt, 1)
    g, gf, init = normal(n, f, 3, dt), normal(3, f, 4), normal(3, f, 5)
    mid, used = slice(offsets[1], offsets[2]), slice(offsets[0], offsets[-1])
    rest = torch.zeros(n, dtype=torch.bool, device="cuda")
    rest[used] = True
    rest[mid] = False

    def run():
        r = tfg.tfg_gated_recurrence(z, x, off, kind, initial=init)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, initial=init, grad_final=gf)
        return [r.out[rest], b.gate[rest], b.x[rest], r.final[[0, 2]], b.initial[[0, 2]]]

    want = run()
    assert all(bool(torch.isfinite(t).all()) for t in want)
    for t in (z, x, g):
        t[:offsets[0]] = float("nan")
        t[offsets[-1]:] = float("inf")
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
    for bad in (float("nan"), -float("inf"), float("inf"), -7.5, 95.0):
        z[mid] = bad
        assert all(torch.equal(a, b) for a, b in zip(run(), want)), bad
