"""Distillation from a teacher's top logits against 64-bit forms.

Tolerances are first-order error bounds, formed element by element in 64 bits, u = 2^-24.  With
y = (s - m) / T, e^y is off by (4 + 3 |y|) u of itself (two roundings of y, the hardware's exponential
within 2 ulp; below 2^-126 it is 0).  The sum's chains hold V / 512 values of a thread (V / 32 in a
warp's rows, up to 8 KB) and 64 more, K = (64 + V / 512 or 32) u, so q is off by
  eq = q ((4 + 3 |y|) u + w + K + 4 u),   w = sum_v q (4 + 3 |y|) u
log p is a difference of (t - t_max) / T and the log of a sum of k terms: el = 4 u (|t - t_max| / T + log k +
4) + k u; p = exp(log p): ep = p (el + 4 u).  Then
  grad: |f| (eq + ep + 4 u (q + p)) + 1e-37 |f|,   f = w T times the loss's gradient
  loss: w T^2 sum_k [ep |log p - log q| + p (el + 4 u |y| + w + K + 4 u (|log p| + |log q|))] + (k + 8) u of
  the sum of |terms|
A gradient stored in bf16 adds half a step, 2^-8 of it.
"""
import gc
import math

import pytest
import torch

from paper_2101_11552_gb300 import tfg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()
    yield
    gc.collect()                                             # exceptions that tests kept, and the tensors in their frames
    torch.cuda.empty_cache()


def close(got, want, tol, what):
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    off = (got.double() - want).abs()
    bad = ~((off <= tol) | (got.double() == want))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {(off / tol.clamp(min=1e-300)).max():.3g} of the bound, first {bad.nonzero()[:3].tolist()}"


class Plain:
    def __init__(self, logits, ids, teacher, tau, weight, padding=-1):
        n, v = logits.shape
        k = ids.shape[1]
        ids = ids.long()
        w = torch.ones(n, device="cuda").double() if weight is None else weight.double()
        here = (ids != padding) & (ids >= 0) & (ids < v)
        at = torch.where(here, ids, 0)
        t = torch.where(here, teacher.double() / tau, -INF)
        self.live = (t.max(1).values > -INF) & (w != 0)
        y = logits.double() / tau
        y = torch.where(self.live[:, None], y - y.max(1, keepdim=True).values, 0.0)
        log_sum = torch.logsumexp(y, 1, keepdim=True)
        q = torch.exp(y - log_sum)
        ry = torch.where(q > 0, (4 + 3 * y.abs()) * U, 0.0)
        wide = (q * ry).sum(1, keepdim=True)
        kk = (64 + v / (32 if v * logits.element_size() <= 8192 else 512)) * U
        eq = q * (ry + wide + kk + 4 * U)
        top = torch.where(self.live[:, None], t, 0.0)
        log_p = torch.log_softmax(torch.where(here & self.live[:, None], top, -INF), 1)
        log_p = torch.where(here & self.live[:, None], log_p, -INF)
        p = torch.where(log_p > -INF, log_p.exp(), 0.0)
        gap = torch.where(p > 0, (top.max(1, keepdim=True).values - top).abs(), 0.0)
        el = 4 * U * (gap + math.log(k) + 4) + k * U
        ep = p * (el + 4 * U)
        yk = torch.where(p > 0, y.gather(1, at), 0.0)
        log_q = yk - log_sum
        lp = torch.where(p > 0, log_p, 0.0)
        terms = torch.where(p > 0, p * (lp - log_q), 0.0)
        live = self.live.double()
        wt = torch.where(self.live, w, 0.0)
        self.loss = wt * tau ** 2 * torch.where(self.live, terms.sum(1), 0.0)
        per = ep * (lp - log_q).abs() + p * (el + 4 * U * yk.abs() + wide + kk + 4 * U * (lp.abs() + log_q.abs()))
        self.loss_tol = live * wt.abs() * tau ** 2 * (torch.where(p > 0, per, 0.0).sum(1) + (k + 8) * U * terms.abs().sum(1))
        full = torch.zeros_like(q).scatter_add_(1, at, torch.where(here, p, 0.0))
        full_tol = torch.zeros_like(q).scatter_add_(1, at, torch.where(here, ep, 0.0))
        self.f = (wt * tau)[:, None]
        self.slope = torch.where(self.live[:, None], q - full, 0.0)
        self.slope_tol = live[:, None] * (eq + full_tol + (4 + k) * U * (q + full) + 1e-37)

    def grad(self, upstream=None):
        f = self.f if upstream is None else self.f * upstream.double()[:, None]
        return f * self.slope, f.abs() * self.slope_tol


def make(n, v, k, seed, dt="f32", tdt="f32", id64=True, spread=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    logits = spread * torch.randn(n, v, device="cuda", generator=gen)
    ids = torch.rand(n, v, device="cuda", generator=gen).argsort(1)[:, :k].contiguous() if v <= 4096 else \
        torch.randint(0, v, (n, k), device="cuda", generator=gen)
    teacher = 3.0 + 2.0 * torch.randn(n, k, device="cuda", generator=gen)
    logits.scatter_add_(1, ids, 0.5 * teacher)
    return logits.to(DT[dt]), ids if id64 else ids.int(), teacher.to(DT[tdt])


def check(logits, ids, teacher, tau=1.0, weight=None, padding=-1, upstream=None):
    p = Plain(logits, ids, teacher, tau, weight, padding)
    a = dict(temperature=tau, row_weight=weight, padding_id=padding)
    r = tfg.tfg_distillation_loss(logits, ids, teacher, **a, want_grad=True, want_stats=True)
    tfg.check_status(r.status)
    close(r.loss, p.loss, p.loss_tol, "loss")
    close(r.grad_logits, *p.grad(), "gradient")
    alone = tfg.tfg_distillation_loss(logits, ids, teacher, **a)
    assert torch.equal(alone.loss, r.loss) and alone.grad_logits is None and alone.stats is None
    if upstream is None:
        upstream = torch.linspace(-1, 2, logits.shape[0], device="cuda")
    back = tfg.tfg_distillation_loss_backward(logits, ids, teacher, tau, r.stats, upstream, row_weight=weight, padding_id=padding)
    close(back, *p.grad(upstream), "backward")
    return r


CLASSES = [1, 2, 3, 5, 7, 8, 16, 31, 32, 33, 41, 64, 100, 255, 256, 1000, 1024, 2047, 2048, 2049, 2056, 4095, 4096, 4097, 4104, 5000, 16_384, 50_001]


@pytest.mark.parametrize("v", CLASSES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_classes(v, dt):
    for n, k in ((1, 1), (9, min(v, 6))):
        check(*make(n, v, k, v, dt, "bf16", id64=v % 2 == 0))


@pytest.mark.parametrize("v", [1, 2, 5, 7, 8, 15, 33, 41, 64, 100, 127, 128, 129])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [9_729, 12_003])
def test_many_rows_of_few_classes(v, dt, n):
    """Rows that share a warp, rows that count for nothing between them, and the last warp's rows that are not there."""
    logits, ids, teacher = make(n, v, min(v, 32), v, dt, "f32", id64=v % 2 == 0)
    weight = torch.linspace(0.5, 2.0, n, device="cuda")
    weight[::7] = 0.0
    logits[::7] = math.nan
    ids[3::11] = -1
    ids[5::13, ::2] = -1
    logits[3::11] = math.inf
    guard = torch.full((n * v + 64,), 9.0, dtype=DT[dt], device="cuda")
    r = check(logits, ids, teacher, 2.0, weight)
    assert not bool(r.loss[::7].any()) and not bool(r.grad_logits[3::11].any())
    grad = guard[32:32 + n * v].view(n, v)                   # on the boundary where the logits are
    again = tfg.tfg_distillation_loss(logits, ids, teacher, temperature=2.0, row_weight=weight, grad_logits=grad)
    assert torch.equal(again.loss, r.loss) and torch.equal(grad, r.grad_logits)
    assert bool((guard[:32] == 9).all()) and bool((guard[32 + n * v:] == 9).all()), "values beside the gradient are left"
    grad = guard[33:33 + n * v].view(n, v)
    odd = tfg.tfg_distillation_loss(logits, ids, teacher, temperature=2.0, row_weight=weight, grad_logits=grad)
    p = Plain(logits, ids, teacher, 2.0, weight)
    close(odd.loss, p.loss, p.loss_tol, "loss")
    close(grad, *p.grad(), "gradient off the boundary")


@pytest.mark.parametrize("v,k", [(128, 128), (200, 129), (2048, 128), (1024, 1024), (2500, 1024), (60_000, 300), (41, 41)])
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
def test_top_sizes_and_temperatures(v, k, tau):
    check(*make(5, v, k, k, "f32", "f32"), tau=tau)


@pytest.mark.parametrize("v,dt", [(120_000, "bf16"), (131_072, "bf16"), (56_000, "f32"), (60_001, "f32"), (300_000, "bf16"), (500_003, "bf16"),
                                  (1_000_000, "f32")])
def test_long_rows(v, dt):
    check(*make(4, v, 20, 3, dt, "f32"), tau=2.0)


@pytest.mark.parametrize("n", [0, 1, 7, 8, 9, 153, 1000])
@pytest.mark.parametrize("v", [41, 3000])
def test_row_counts(n, v):
    logits, ids, teacher = make(n, v, 5, n + 1)
    if n == 0:
        r = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True, want_stats=True)
        assert r.loss.shape == (0,) and int(r.status) == 0
        assert tfg.tfg_distillation_loss_backward(logits, ids, teacher, 1.0, r.stats, r.loss).shape == (0, v)
        return
    check(logits, ids, teacher)


@pytest.mark.parametrize("v", [41, 5000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_padding_weights_and_empty_rows(v, dt):
    logits, ids, teacher = make(40, v, 6, 1, dt)
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids[torch.rand(40, 6, device="cuda", generator=gen) < 0.3] = -1
    ids[3] = -1                                              # nothing of the teacher
    teacher[5] = -INF
    teacher[6, 1:] = -INF
    weight = torch.rand(40, device="cuda", generator=gen) - 0.3
    weight[7] = 0.0
    logits[7] = float("nan")                                 # not read
    logits[3, 0] = INF
    r = check(logits, ids, teacher, 1.5, weight)
    for row in (3, 5, 7):
        assert float(r.loss[row]) == 0.0 and bool((r.grad_logits[row] == 0).all()) and r.stats[row].tolist() == [0.0, 1.0]


@pytest.mark.parametrize("padding", [0, 40, -(1 << 63), (1 << 63) - 1])
@pytest.mark.parametrize("id64", [True, False])
def test_padding_ids(padding, id64):
    logits, ids, teacher = make(30, 41, 6, 1, id64=id64)
    check(logits, ids, teacher, padding=padding)


@pytest.mark.parametrize("v,k", [(41, 12), (6000, 40), (6000, 200)])
def test_a_class_listed_more_than_once(v, k):
    logits, ids, teacher = make(20, v, k, 4)
    ids[:, 1::3] = ids[:, :1]
    ids[:, -1] = ids[:, 2]
    check(logits, ids, teacher, 2.0)


@pytest.mark.parametrize("v", [41, 5000])
def test_masked_classes(v):
    """Logits of -inf: no probability and no gradient; an infinite loss where the teacher has some."""
    logits, ids, teacher = make(12, v, 4, 1)
    logits[0::2, v // 2] = -INF
    ids[0::2][ids[0::2] == v // 2] = -1
    r = check(logits, ids, teacher)
    assert bool((r.grad_logits[0::2, v // 2] == 0).all())
    logits[1, ids[1, 0]] = -INF
    r = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True)
    assert float(r.loss[1]) == INF and bool(torch.isfinite(r.grad_logits[1]).all()) and float(r.grad_logits[1, ids[1, 0]]) < 0
    teacher[1, 0] = -INF                                     # 0 times infinity is nothing here
    r = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True)
    assert math.isfinite(float(r.loss[1]))


@pytest.mark.parametrize("v", [41, 5000])
def test_numbers_that_are_none_stay_in_their_row(v):
    logits, ids, teacher = make(20, v, 4, 1)
    want = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True)
    logits[2, 7], logits[4, 9] = float("nan"), INF
    logits[6] = -INF
    teacher[8, 1], teacher[10, 2] = float("nan"), INF
    teacher[12] = float("nan")
    ids[12, 1:] = -1
    got = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True, padding_id=-1)
    bad = [2, 4, 6, 8, 10, 12]
    rest = [i for i in range(20) if i not in bad]
    assert torch.equal(got.loss[rest], want.loss[rest]) and torch.equal(got.grad_logits[rest], want.grad_logits[rest])
    for i in bad:
        assert bool(torch.isnan(got.loss[i])) and bool(torch.isnan(got.grad_logits[i]).any()), i


def test_large_offset():
    """Logits that share an offset of 4,096 lose nothing: s - m is exact."""
    logits, ids, teacher = make(16, 3000, 8, 1)
    logits = (logits * 16).round() / 16                      # sums with the offset are exact
    want = tfg.tfg_distillation_loss(logits, ids, teacher, want_grad=True)
    got = tfg.tfg_distillation_loss(logits + 4096.0, ids, teacher, want_grad=True)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.grad_logits, want.grad_logits)


def test_a_student_that_knows_the_teacher():
    """Equal distributions over all classes: a loss and a gradient of nothing but rounding."""
    teacher = torch.randn(10, 100, device="cuda")
    ids = torch.arange(100, device="cuda").expand(10, 100).contiguous()
    r = check(teacher.clone(), ids, teacher, 2.0)
    assert bool((r.loss.abs() <= 1e-5).all()) and bool((r.grad_logits.abs() <= 1e-6).all())


@pytest.mark.parametrize("by", [1, 2, 3, 8])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("v", [41, 4999])
def test_offset_pointers(by, dt, v):
    """Logits and gradients off each other's 16-byte boundaries."""
    logits, ids, teacher = make(7, v, 5, 1, dt)
    want = check(logits, ids, teacher)
    for lb, gb in ((by, by), (by, 0), (0, by)):
        a, b = (torch.full((7 * v + 32,), 5.0, dtype=DT[dt], device="cuda") for _ in range(2))
        moved, grad = a[lb:lb + 7 * v].view(7, v), b[gb + 8:gb + 8 + 7 * v].view(7, v)
        moved.copy_(logits)
        r = tfg.tfg_distillation_loss(moved, ids, teacher, want_stats=True, grad_logits=grad)
        p = Plain(logits, ids, teacher, 1.0, None)
        close(r.loss, p.loss, p.loss_tol, "loss")
        close(grad, *p.grad(), "gradient")
        assert bool((b[:gb + 8] == 5).all()) and bool((b[gb + 8 + 7 * v:] == 5).all()), "nothing beside the gradient is written"
    assert want.grad_logits.shape == (7, v)


@pytest.mark.parametrize("n", [3, 9000])
@pytest.mark.parametrize("bad", [41, -2, 1 << 30])
@pytest.mark.parametrize("id64", [True, False])
def test_ids_outside_are_reported(n, bad, id64):
    logits, ids, teacher = make(n, 41, 4, 1, id64=id64)
    want = ids.clone()
    want[n // 2, 2] = -1
    ids[n // 2, 2] = bad
    r = tfg.tfg_distillation_loss(logits, ids, teacher, padding_id=-1, want_grad=True, want_stats=True)
    assert int(r.status) == tfg.TFG_ERR_INDEX_RANGE
    ref = tfg.tfg_distillation_loss(logits, want, teacher, padding_id=-1, want_grad=True)
    assert int(ref.status) == 0 and torch.equal(r.loss, ref.loss) and torch.equal(r.grad_logits, ref.grad_logits)
    back = tfg.tfg_distillation_loss_backward(logits, ids, teacher, 1.0, r.stats, torch.ones(n, device="cuda"), padding_id=-1)
    assert bool(torch.isfinite(back).all())


def test_gradient_is_the_slope():
    logits, ids, teacher = make(6, 30, 4, 1)
    w = torch.linspace(0.2, 1.5, 6, device="cuda")
    tau = 1.7

    def loss(s):
        log_p = torch.log_softmax(teacher.double() / tau, 1)
        log_q = torch.log_softmax(s / tau, 1).gather(1, ids)
        return float((w.double() * tau ** 2 * (log_p.exp() * (log_p - log_q)).sum(1)).sum())

    r = tfg.tfg_distillation_loss(logits, ids, teacher, tau, row_weight=w, want_grad=True)
    u = torch.randn(6, 30, device="cuda", dtype=torch.float64)
    slope = (loss(logits.double() + 1e-4 * u) - loss(logits.double() - 1e-4 * u)) / 2e-4
    assert abs(slope - float((r.grad_logits.double() * u).sum())) <= 1e-5 * float(r.grad_logits.double().norm() * u.norm())


def test_refusals():
    logits, ids, teacher = make(4, 20, 3, 1)
    for bad in (dict(logits=logits.t()), dict(ids=ids[:3]), dict(teacher=teacher[:, :2]), dict(logits=logits.half()),
                dict(row_weight=torch.ones(3, device="cuda")), dict(padding_id=1 << 63), dict(logits=logits.cpu()),
                dict(grad_logits=torch.empty(4, 20, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            tfg.tfg_distillation_loss(**{**dict(logits=logits, ids=ids, teacher=teacher), **bad})
    with pytest.raises(TypeError):
        tfg.tfg_distillation_loss(logits, ids.short(), teacher)
    for tau in (0.0, -1.0, INF, float("nan"), 1e-7, 1e7):
        with pytest.raises(tfg.TfgError):
            tfg.tfg_distillation_loss(logits, ids, teacher, tau)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_distillation_loss(logits, ids, teacher, grad_logits=logits)
    with pytest.raises(tfg.TfgError) as e:
        tfg.tfg_distillation_loss(torch.zeros(2, 3000, device="cuda"), torch.zeros(2, 1025, dtype=torch.int64, device="cuda"),
                                  torch.zeros(2, 1025, device="cuda"))
    assert e.value.code == tfg.TFG_ERR_TOO_LARGE
    with pytest.raises(ValueError):
        tfg.tfg_distillation_loss_backward(logits, ids, teacher, 1.0, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"))
