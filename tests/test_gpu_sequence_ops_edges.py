"""Calls that the documentation of the layer-norm, recurrence and distillation entry points allows and that
ordinary batches do not make: rows apart by odd strides, arrays of more than 2^31 values, calls from
several threads, more teacher entries than classes, statuses that earlier calls left."""
import gc
import threading

import pytest
import torch

from paper_2101_11552_gb300 import build, tfg
from test_gpu_distillation import check as check_distillation
from test_gpu_gated_recurrence import Plain, batch, check as check_recurrence, close, normal
from test_gpu_layer_norm import check as check_norm, features

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    yield
    gc.collect()                                             # exceptions that tests kept, and the tensors in their frames
    torch.cuda.empty_cache()


def apart(t, ld, first):
    """t's rows ld values apart in a buffer of their own, from value `first` on."""
    n, f = t.shape
    buf = torch.zeros(n * ld + first + 16, dtype=t.dtype, device="cuda")
    v = buf[first:first + n * ld].view(n, ld)[:, :f]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("f,ld,first", [(32, 33, 0), (32, 48, 1), (32, 48, 8), (8, 200, 0), (40, 41, 3), (64, 72, 4)])
def test_rows_apart(dt, f, ld, first):
    offsets = [0, 150, 151, 400]
    z, x = batch(400, f, "sigmoid", dt, 1)
    check_recurrence(apart(z, ld, first), apart(x, ld + 8, first), offsets, "sigmoid", normal(3, f, 2), dt, normal(400, f, 3, dt),
                     normal(3, f, 4))


def test_one_row_of_any_stride():
    z, x = batch(1, 16, "exp", "f32", 1)
    off = torch.tensor([0, 1], device="cuda")
    want = tfg.tfg_gated_recurrence(z, x, off, "exp").out
    wide = torch.zeros(1, 1 << 20, device="cuda")
    wide[:, :16] = z
    assert torch.equal(tfg.tfg_gated_recurrence(wide[:, :16], x, off, "exp").out, want)


@pytest.mark.parametrize("aligned", [True, False])
def test_recurrence_over_more_than_2_31_values(aligned):
    """The last sequence of a batch whose values pass 32 bits, against the same rows by themselves.  It begins a
    tile and a window, so that the same maps are composed in the same order."""
    f = 1024 if aligned else 1023
    n, tail = (1 << 21) + 4096 * 3, 4096 + 300
    n -= n % 4096
    first = n - 8192
    z = torch.full((n, f), 2.0, dtype=torch.bfloat16, device="cuda")
    x = torch.ones_like(z)
    zt, xt = batch(tail, f, "sigmoid", "bf16", 1)
    z[first:first + tail], x[first:first + tail] = zt, xt
    off = torch.tensor([0, first, first + tail], device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off)
    tfg.check_status(r.status)
    alone = tfg.tfg_gated_recurrence(zt, xt, torch.tensor([0, tail], device="cuda"))
    assert torch.equal(r.out[first:first + tail], alone.out) and torch.equal(r.final[1], alone.final[0])
    # rows of equal inputs approach their input of 1 (in fp32 within 1e-6 after 200 rows of a = 0.88)
    assert bool((r.out[1000:first:997].float() == 1.0).all())
    g = torch.zeros(n, f, dtype=torch.bfloat16, device="cuda")
    gt = normal(tail, f, 3, "bf16")
    g[first:first + tail] = gt
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, want_initial=True)
    p = tfg.tfg_gated_recurrence_backward(zt, xt, off[:2] * 0 + torch.tensor([0, tail], device="cuda"), alone.checkpoints, gt,
                                          want_initial=True)
    # the order of work runs from the last row, so windows lie otherwise: within the rounding of bf16
    for got, want in ((b.gate[first:first + tail], p.gate), (b.x[first:first + tail], p.x)):
        assert float((got.float() - want.float()).norm()) <= 2.0 ** -8 * float(want.float().norm())
    assert bool((b.gate[:first:1013] == 0).all()) and bool((b.x[first + tail - 1].isfinite()).all())


def test_layer_norm_over_more_than_2_31_values():
    n, f = (1 << 21) + 5, 1024
    x = torch.zeros(n, f, dtype=torch.bfloat16, device="cuda")
    tail = features(5, f, 1, "bf16")
    x[-5:] = tail
    r = tfg.tfg_layer_norm(x)
    want = tfg.tfg_layer_norm(tail)
    assert torch.equal(r.out[-5:], want.out) and bool((r.out[:-5:1009] == 0).all())
    g = torch.zeros_like(x)
    g[-5:] = features(5, f, 2, "bf16")
    gx, gg, gb = tfg.tfg_layer_norm_backward(x, None, r.mean, r.rstd, g)
    wx, wg, wb = tfg.tfg_layer_norm_backward(tail, None, want.mean, want.rstd, g[-5:].clone())
    assert torch.equal(gx[-5:], wx) and bool((gx[:-5:1009] == 0).all())
    # five rows that are not 0, in another order
    assert bool(((gg - wg).abs() <= 1e-5 * (1 + wg.abs())).all()) and bool(((gb - wb).abs() <= 1e-5 * (1 + wb.abs())).all())


def test_distillation_over_more_than_2_31_values():
    n, v, k = 43_000, 50_000, 4
    logits = torch.zeros(n, v, dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(n * k, device="cuda").reshape(n, k) % v
    teacher = torch.randn(n, k, device="cuda")
    logits[-3:] = torch.randn(3, v, device="cuda").bfloat16()
    r = tfg.tfg_distillation_loss(logits, ids, teacher, 2.0, want_grad=True, want_stats=True)
    want = tfg.tfg_distillation_loss(logits[-3:], ids[-3:], teacher[-3:], 2.0, want_grad=True, want_stats=True)
    tfg.check_status(r.status)
    assert torch.equal(r.loss[-3:], want.loss) and torch.equal(r.grad_logits[-3:], want.grad_logits)
    back = tfg.tfg_distillation_loss_backward(logits, ids, teacher, 2.0, r.stats, torch.ones(n, device="cuda"))
    assert torch.equal(back[-3:], tfg.tfg_distillation_loss_backward(logits[-3:], ids[-3:], teacher[-3:], 2.0, want.stats,
                                                                     torch.ones(3, device="cuda")))


@pytest.mark.parametrize("v,k", [(3, 10), (50, 200), (700, 1024)])
def test_more_teacher_entries_than_classes(v, k):
    gen = torch.Generator(device="cuda").manual_seed(v)
    check_distillation(torch.randn(7, v, device="cuda", generator=gen), torch.randint(0, v, (7, k), device="cuda", generator=gen),
                       torch.randn(7, k, device="cuda", generator=gen), 1.5)


@pytest.mark.parametrize("v", [1000, 5000, 20_000, 45_000, 60_000, 130_000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_a_loss_has_the_same_bits_with_its_gradient(v, dt):
    """Many rows, a third of them masked, one without teacher: loss alone, with gradient, in two calls."""
    n, k = 700, 9
    gen = torch.Generator(device="cuda").manual_seed(v)
    logits = (2 * torch.randn(n, v, device="cuda", generator=gen)).to(dt)
    ids = torch.randint(0, v, (n, k), device="cuda", generator=gen).int()
    ids[5] = -1
    teacher = torch.randn(n, k, device="cuda", generator=gen)
    w = (torch.rand(n, device="cuda", generator=gen) > 0.33).float()
    a = dict(row_weight=w, padding_id=-1)
    alone = tfg.tfg_distillation_loss(logits, ids, teacher, 1.5, **a)
    both = tfg.tfg_distillation_loss(logits, ids, teacher, 1.5, **a, want_grad=True, want_stats=True)
    assert torch.equal(alone.loss, both.loss)
    again = tfg.tfg_distillation_loss(logits, ids, teacher, 1.5, **a, want_grad=True)
    assert torch.equal(again.grad_logits, both.grad_logits)
    back = tfg.tfg_distillation_loss_backward(logits, ids, teacher, 1.5, both.stats, torch.ones(n, device="cuda"), **a)
    assert torch.equal(back, both.grad_logits)
    assert bool((both.grad_logits[w == 0] == 0).all()) and float(both.loss[5]) == 0.0


def test_statuses_are_written_anew():
    z, x = batch(300, 32, "sigmoid", "f32", 1)
    good, bad = torch.tensor([0, 300], device="cuda"), torch.tensor([0, 400], device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = tfg.tfg_gated_recurrence(z, x, good).checkpoints
    for off, want in ((bad, tfg.TFG_ERR_INDEX_RANGE), (good, 0), (bad, tfg.TFG_ERR_INDEX_RANGE), (good, 0)):
        tfg.tfg_gated_recurrence_backward(z, x, off, kept, x, status=word)
        assert int(word) == want


def test_from_several_threads():
    """Calls of different sizes from threads of their own, each on its own stream."""
    jobs = []
    for i, (n, f, cuts) in enumerate([(9000, 128, [0, 9000]), (3000, 33, [0, 5, 2000, 3000]), (100, 64, list(range(101)))]):
        z, x = batch(n, f, "sigmoid", "bf16", i)
        jobs.append((z, x, torch.tensor(cuts, device="cuda"), normal(n, f, 9, "bf16"), normal(f, 1, 8).flatten()))

    def step(z, x, off, g, gamma):
        r = tfg.tfg_gated_recurrence(z, x, off)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g)
        h = tfg.tfg_layer_norm(r.out, gamma, None, residual=x)
        gx = tfg.tfg_layer_norm_backward(h.sum, gamma, h.mean, h.rstd, g)
        ids = torch.zeros(z.shape[0], 1, dtype=torch.int64, device="cuda")
        d = tfg.tfg_distillation_loss(h.out, ids, g[:, :1].float().contiguous(), want_grad=True)
        return [r.out, r.final, b.gate, b.x, h.out, *gx, d.loss, d.grad_logits]

    alone = [step(*j) for j in jobs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(25):
                    got = step(*jobs[i])
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, alone[i])):
                    wrong.append(i)
        except Exception as e:                               # seen by the main thread
            wrong.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_long_recurrences_beside_one_another():
    """Two streams whose kernels each want the whole device, with workspaces of their own."""
    z, x = batch(60_000, 512, "sigmoid", "bf16", 1)
    offs = [torch.tensor(c, device="cuda") for c in ([0, 60_000], [0, 11, 30_000, 60_000])]
    want = [tfg.tfg_gated_recurrence(z, x, o) for o in offs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in offs]
    got = []
    for _ in range(6):
        for s, o in zip(streams, offs):
            with torch.cuda.stream(s):
                got.append(tfg.tfg_gated_recurrence(z, x, o))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert int(r.status) == 0 and torch.equal(r.out, want[i % 2].out) and torch.equal(r.final, want[i % 2].final)


@pytest.mark.parametrize("f", [64, 256, 1024, 2048, 4096, 8192])
@pytest.mark.parametrize("n", [1, 31, 33, 1217, 3001])
def test_norm_rows_beside_the_teams(f, n):
    """Counts of rows around the teams, units and CTAs of the backward, in mixed types."""
    check_norm(features(n, f, 1, "bf16"), features(n, f, 2, "f32"), torch.linspace(0.5, 1.5, f, device="cuda"), None, "bf16",
               features(n, f, 3, "bf16"), features(n, f, 4, "f32"))


def test_recurrence_states_of_a_chain_of_calls():
    """Ten calls, each continuing the last, eager and with the states' gradients handed back, against one call."""
    n, f, parts = 1000, 40, 10
    z, x = batch(n, f, "exp", "f32", 1)
    g = normal(n, f, 2)
    step = n // parts
    cut = torch.tensor([0, step], device="cuda")
    runs, state = [], None
    for i in range(parts):
        r = slice(i * step, (i + 1) * step)
        runs.append((r, state, tfg.tfg_gated_recurrence(z[r], x[r], cut, "exp", initial=state)))
        state = runs[-1][2].final
    p = Plain(z, x, [0, n], "exp", None)
    for r, _, run in runs:
        close(run.out, p.v[r], p.e[r], "out")
    (wz, tz), (wx, tx), _ = p.backward(g, None)
    last = None
    for r, state, run in reversed(runs):
        b = tfg.tfg_gated_recurrence_backward(z[r], x[r], cut, run.checkpoints, g[r], "exp", initial=state, grad_final=last, want_initial=True)
        close(b.gate, wz[r], tz[r], "grad_gate")
        close(b.x, wx[r], tx[r], "grad_x")
        last = b.initial
