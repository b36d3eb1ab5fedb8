"""Layer norm of rows with a residual stream, forward and backward, against 64-bit forms.

Tolerances are first-order error bounds, formed element by element in 64 bits, u = 2^-24.  A
thread adds at most 64 values of a row by itself (rows that no team holds: F / 1024 partial
sums), butterflies and a warp's worth of partial sums follow, so a mean of terms t is off by
at most K mean |t|, K = (128 + F / 1024) u.  With c = s - m, D = mean |c| + K mean |s| (deviations
from a first mean that is off by K mean |s|) the centred value is off by
  ec = K D + 2 u (|c| + K mean |s|),   dr / r <= (K + 4 u) / 2 + (K D r)^2 + 4 u
  eh = r ec + |h| (dr / r + 2 u),   out: |gamma| eh + 3 u (|gamma h| + |beta|)
Backward, with the reported mean off by another u |m| (e = r u |m| at most, taken out again with an
error of K r mean |c'|, |c'| <= |c| + u |m|):
  eh' = r (K (mean |c| + u |m|) + 2 u (|c| + u |m|)) + |h| (dr / r + 2 u)
  s1 = mean d: K mean |d|;   s2 = mean d h: mean(|d| eh') + (K + 4 u) mean |d| (|h| + e) + 2 e K mean |d|
  grad_s: r (3 u |d| + es1 + |h| es2 + |s2| eh') + r (|d| + |s1| + |h s2|) (dr / r + 6 u) + 2 u |grad_sum|
  columns: sums over rows in chains of N / CTAs, 32 teams and the CTAs in 32 chains, at most
  Kn = (N + 120) u of sum |t| whatever the split; terms off by |g| eh'.
A result stored in bf16 adds half a step, 2^-8 of it.
"""
import gc
import pytest
import torch

from paper_2101_11552_gb300 import tfg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


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
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {(off / tol.clamp(min=1e-300)).max():.3g} of the bound"


class Plain:
    def __init__(self, s, gamma, beta, eps=EPS):
        self.n, self.f = s.shape
        k = self.k = (128 + self.f / 1024) * U
        s = s.double()
        self.gamma = torch.ones(self.f, device=s.device).double() if gamma is None else gamma.double()
        beta = torch.zeros(self.f, device=s.device).double() if beta is None else beta.double()
        self.mean = s.mean(1, keepdim=True)
        self.c = s - self.mean
        var = (self.c ** 2).mean(1, keepdim=True)
        self.r = (var + eps) ** -0.5
        away = k * s.abs().mean(1, keepdim=True)
        d = self.c.abs().mean(1, keepdim=True) + away
        self.rel = (k + 4 * U) / 2 + (k * d * self.r) ** 2 + 4 * U
        ec = k * d + 2 * U * (self.c.abs() + away)
        self.h = self.c * self.r
        eh = self.r * ec + self.h.abs() * (self.rel + 2 * U)
        self.out = self.h * self.gamma + beta
        self.out_tol = self.gamma.abs() * eh + 3 * U * ((self.gamma * self.h).abs() + beta.abs())
        self.mean_tol = k * d + 2 * U * self.mean.abs()

    def backward(self, g, skip):
        g = g.double()
        k, r, h = self.k, self.r, self.h
        shift = U * self.mean.abs()
        eh = r * (k * (self.c.abs().mean(1, keepdim=True) + shift) + 2 * U * (self.c.abs() + shift)) \
            + h.abs() * (self.rel + 2 * U)
        e = r * shift
        d = g * self.gamma
        s1, s2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
        size = d.abs().mean(1, keepdim=True)
        es1 = k * size
        es2 = (d.abs() * eh).mean(1, keepdim=True) + (k + 4 * U) * (d.abs() * (h.abs() + e)).mean(1, keepdim=True) + 2 * e * k * size
        gs = r * (d - s1 - h * s2)
        tol = r * (3 * U * d.abs() + es1 + h.abs() * es2 + s2.abs() * eh) \
            + r * (d.abs() + s1.abs() + (h * s2).abs()) * (self.rel + 6 * U)
        if skip is not None:
            gs = gs + skip.double()
            tol = tol + 2 * U * (skip.double().abs() + gs.abs())
        kn = (self.n + 120) * U
        gg = ((g * h).sum(0), (g.abs() * eh).sum(0) + kn * (g * h).abs().sum(0))
        return (gs, tol), gg, (g.sum(0), kn * g.abs().sum(0))


def features(n, f, seed, dtype, spread=1.0, offset=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = spread * torch.randn(n, f, device="cuda", generator=gen) + offset * torch.randn(n, 1, device="cuda", generator=gen)
    return x.to(DT[dtype])


def check(x, res, gamma, beta, out_dtype, g, skip=None, grad_dtype=None):
    r = tfg.tfg_layer_norm(x, gamma, beta, EPS, residual=res, out_dtype=DT[out_dtype])
    if res is None:
        assert r.sum is x
    else:
        assert torch.equal(r.sum, (x.double() + res.double()).to(res.dtype)), "the sum is rounded once"
    p = Plain(r.sum, gamma, beta)
    close(r.out, p.out, p.out_tol, "out")
    close(r.mean[:, None], p.mean, p.mean_tol, "mean")
    close(r.rstd[:, None], p.r, p.r * p.rel, "rstd")
    gx, gg, gb = tfg.tfg_layer_norm_backward(r.sum, gamma, r.mean, r.rstd, g, grad_sum=skip, grad_dtype=grad_dtype)
    (ws, ts), (wg, tg), (wb, tb) = p.backward(g, skip)
    close(gx, ws, ts, "grad_x")
    close(gg, wg, tg, "grad_gamma")
    close(gb, wb, tb, "grad_beta")
    return r, (gx, gg, gb)


WIDTHS = [1, 2, 3, 7, 8, 12, 31, 32, 33, 64, 72, 100, 123, 128, 255, 256, 257, 264, 512, 520, 1000, 1024, 1032, 2047, 2048, 2056,
          4096, 4104, 8192, 8200, 16384, 16392, 32768]


@pytest.mark.parametrize("f", WIDTHS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_widths(f, dt):
    for n in (1, 37):
        gen = torch.Generator(device="cuda").manual_seed(f)
        gamma, beta = 1 + 0.2 * torch.randn(2, f, device="cuda", generator=gen)
        check(features(n, f, f + n, dt), features(n, f, f + n + 1, dt), gamma, beta, dt, features(n, f, 3, dt),
              features(n, f, 4, dt))
        check(features(n, f, f + n, dt), None, None, None, dt, features(n, f, 3, dt))


@pytest.mark.parametrize("f", [1023, 1025, 1032, 2047, 2048, 2052, 2056, 4092, 4096, 4100, 4104, 8188, 8192, 8196, 8200, 16376, 16384,
                               16388, 16392, 32764, 32768])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_widths_around_the_wide_teams(f, dt):
    n = 700 if f <= 2056 else 23
    check(features(n, f, 1, "bf16"), features(n, f, 2, dt), torch.linspace(0.5, 1.5, f, device="cuda"),
          torch.linspace(-1, 1, f, device="cuda"), dt, features(n, f, 3, dt), features(n, f, 4, dt))


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("res", [None, "f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("f", [96, 123, 2048])
def test_types(x, res, out, f):
    n = 301
    gamma = torch.linspace(0.5, 1.5, f, device="cuda")
    beta = torch.linspace(-1, 1, f, device="cuda")
    for grad in ("f32", "bf16"):
        skip = None if res is None else features(n, f, 5, grad)
        check(features(n, f, 1, x), None if res is None else features(n, f, 2, res), gamma, beta, out, features(n, f, 4, out),
              skip, None if skip is not None else DT[grad])


@pytest.mark.parametrize("f,dt", [(32776, "f32"), (40001, "f32"), (40001, "bf16"), (65536, "bf16"), (100_004, "f32")])
def test_rows_that_no_team_holds(f, dt):
    n = 9
    gamma = torch.linspace(0.5, 1.5, f, device="cuda")
    r, _ = check(features(n, f, 1, dt), features(n, f, 2, "f32"), gamma, gamma, dt, features(n, f, 3, dt), features(n, f, 4, "f32"))
    gx, gg, gb = tfg.tfg_layer_norm_backward(r.sum, gamma, r.mean, r.rstd, features(n, f, 3, dt), want_weight_grads=False)
    assert gg is None and gb is None and bool(torch.isfinite(gx).all())


@pytest.mark.parametrize("n", [2, 7, 8, 9, 303, 304, 305, 2432, 2433, 20_011])
@pytest.mark.parametrize("f", [40, 128, 1024])
def test_row_counts(n, f):
    check(features(n, f, 1, "f32"), None, torch.linspace(0.5, 1.5, f, device="cuda"), None, "f32", features(n, f, 2, "f32"))


@pytest.mark.parametrize("f", [96, 1000, 9000, 40_000])
@pytest.mark.parametrize("offset,spread", [(1000.0, 1.0), (30000.0, 0.01), (-3.0, 1e-4)])
def test_far_mean(f, offset, spread):
    gen = torch.Generator(device="cuda").manual_seed(f)
    x = offset + spread * torch.randn(11, f, device="cuda", generator=gen)
    check(x, None, None, None, "f32", features(11, f, 2, "f32"))


@pytest.mark.parametrize("f", [1, 5, 64, 1000, 40_000])
def test_equal_values_give_beta(f):
    x = torch.full((5, f), 1234.567, device="cuda")
    check(x, None, None, torch.linspace(-1, 1, f, device="cuda"), "f32", features(5, f, 2, "f32"))


@pytest.mark.parametrize("f", [64, 1000, 8192, 40_000])
def test_offset_pointers(f):
    """Arrays off the vector boundary give what aligned ones give, within the bounds."""
    n = 13
    def moved(t, by):
        buf = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
        v = buf[by:by + t.numel()].view(t.shape)
        v.copy_(t)
        return v
    for by in (1, 2, 4):
        x, res, g, skip = (moved(features(n, f, i, dt), by) for i, dt in enumerate(("bf16", "f32", "bf16", "f32")))
        gamma = moved(torch.linspace(0.5, 1.5, f, device="cuda"), by)
        check(x, res, gamma, gamma, "bf16", g, skip)


@pytest.mark.parametrize("f", [96, 123, 4096, 40_000])
def test_in_place(f):
    n = 50
    x, res, g, skip = (features(n, f, i, dt) for i, dt in enumerate(("bf16", "f32", "bf16", "f32")))
    want = tfg.tfg_layer_norm(x, residual=res)
    stream = res.clone()
    got = tfg.tfg_layer_norm(x, residual=stream, sum_out=stream)
    assert got.sum is stream and torch.equal(stream, want.sum) and torch.equal(got.out, want.out)
    back = tfg.tfg_layer_norm_backward(stream, None, got.mean, got.rstd, g, grad_sum=skip)
    buf = skip.clone()
    again = tfg.tfg_layer_norm_backward(stream, None, got.mean, got.rstd, g, grad_sum=buf, grad_x=buf)
    assert again[0] is buf and all(torch.equal(a, b) for a, b in zip(back, again))


@pytest.mark.parametrize("f", [40, 300, 2000, 40_000])
def test_numbers_that_are_none_stay_in_their_row(f):
    x = features(40, f, 1, "f32")
    clean = tfg.tfg_layer_norm(x)
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"))):
        x[7 * i + 3, f // 2] = v
    rows = [i for i in range(40) if i not in (3, 10, 17)]
    r = tfg.tfg_layer_norm(x)
    assert torch.equal(r.out[rows], clean.out[rows])
    for i in (3, 10, 17):
        assert bool(torch.isnan(r.out[i]).any()) and bool(torch.isnan(r.mean[i]) | torch.isinf(r.mean[i]))
    gx, gg, gb = tfg.tfg_layer_norm_backward(x, None, r.mean, r.rstd, features(40, f, 2, "f32"))
    assert bool(torch.isfinite(gx[rows]).all()) and bool(torch.isnan(gx[3]).all()) and bool(torch.isfinite(gb).all())


def test_no_rows():
    x = torch.empty(0, 24, device="cuda")
    r = tfg.tfg_layer_norm(x, residual=x.clone())
    assert r.out.shape == (0, 24) and r.mean.shape == (0,)
    gx, gg, gb = tfg.tfg_layer_norm_backward(x, None, r.mean, r.rstd, x)
    assert gx.shape == (0, 24) and bool((gg == 0).all()) and bool((gb == 0).all())


def test_gradient_is_the_slope():
    """<grad, u> against central differences of the 64-bit form; the kernel's own error is some
    1e-6 of the gradient, the differences' 1e-8 (step 1e-4, third derivatives of about 1)."""
    n, f = 6, 50
    x, g, gamma = features(n, f, 1, "f32"), features(n, f, 2, "f32"), torch.linspace(0.5, 1.5, f, device="cuda")

    def loss(x, gamma, beta):
        c = x - x.mean(1, keepdim=True)
        return float(((c * ((c ** 2).mean(1, keepdim=True) + EPS) ** -0.5 * gamma + beta) * g.double()).sum())

    r = tfg.tfg_layer_norm(x, gamma, None, EPS)
    grads = tfg.tfg_layer_norm_backward(x, gamma, r.mean, r.rstd, g)
    at = [x.double(), gamma.double(), torch.zeros(f, device="cuda", dtype=torch.float64)]
    for i, grad in enumerate(grads):
        u = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(i))
        plus, minus = ([v + s * 1e-4 * u if j == i else v for j, v in enumerate(at)] for s in (1, -1))
        slope = (loss(*plus) - loss(*minus)) / 2e-4
        assert abs(slope - float((grad.double() * u).sum())) <= 1e-5 * float(grad.double().norm() * u.norm())


def test_refusals():
    x = features(4, 8, 1, "f32")
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x.t())
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x, residual=x[:3])
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x, sum_out=x)
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x, gamma=torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x.double())
    with pytest.raises(tfg.TfgError):
        tfg.tfg_layer_norm(x, out=x)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_layer_norm(x, eps=0.0)
    r = tfg.tfg_layer_norm(x)
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm_backward(x, None, r.mean[:2], r.rstd, x)
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm_backward(x, None, r.mean, r.rstd, x, grad_sum=x.bfloat16(), grad_dtype=torch.float32)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_layer_norm_backward(x, None, r.mean, r.rstd, x, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
