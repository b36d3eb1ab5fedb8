"""Group norm of values far from zero against their spread, forward and backward.

An offset common to all values costs nothing: the deviations from the mean as first found are
summed again, and the mean is used as that sum's correction (rest) says.  Bounds as in
test_gpu_group_norm (u = 2^-24, K = 520 u for a sum), but with c = x - m and v = mean c^2
  rest <= (K + 3 u) 2 max |c| + u |m|     (the first mean: of differences from one of the values,
                                           at most 2 max |c|; and its rounding)
  dm = 2 (K + 3 u) (sqrt(v) + rest)       the error of mean + rest, in place of K mean |x|: that of a
       mean of c - rest, of which the mean absolute value is at most sqrt(v) + rest; twice, as pieces
       of a graph are summed and then joined
  dv = (K + 6 u) (v + rest^2) + 2 rest dm + dm^2 + 4 dm sqrt(v)    the error of the variance: squares
       about the first mean, less the square of the rest; the last term where pieces are joined,
       whose means are off by dm each and at most sqrt(v) from the joint one in the mean
  dr / r <= dv r^2 / 2 + 4 u
  eh = r (dm + u (|c| + rest) + 4 u rest) + |h| (dr / r + 2 u)
The mean is reported, and given to the backward, in fp32: off by u |m| more, and the backward's
eh by r u |m|.
"""
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_group_norm import DT, EPS, K, U, Plain, close, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


class Far(Plain):
    def __init__(self, x, offsets, groups, gamma, beta, act, eps=EPS):
        super().__init__(x, offsets, groups, gamma, beta, act, eps)
        c = x.double()[self.rows] - self.spread(self.mean)
        most = torch.zeros_like(self.mean)
        most.index_reduce_(0, self.graph, c.abs().reshape(c.shape[0], groups, -1).amax(2), "amax")
        v = self.per_graph(c * c)
        rest = (K + 3 * U) * 2 * most + U * self.mean.abs()
        dm = 2 * (K + 3 * U) * (v.sqrt() + rest)
        dv = (K + 6 * U) * (v + rest ** 2) + 2 * rest * dm + dm ** 2 + 4 * dm * v.sqrt()
        self.rel = dv * self.rstd ** 2 / 2 + 4 * U
        r, rest_x = self.spread(self.rstd), self.spread(rest)
        self.eh = r * (self.spread(dm) + U * c.abs() + 5 * U * rest_x) + self.h.abs() * (self.spread(self.rel) + 2 * U)
        self.mean_tol = dm + U * self.mean.abs()
        self.bound()
        self.rounded = r * U * self.spread(self.mean.abs())

    def bound(self):
        self.ey = self.gamma.abs() * self.eh + 2 * U * ((self.gamma * self.h).abs() + self.beta.abs())
        self.out_tol = 1.13 * self.ey + 12 * U * (self.y.abs() + self.out.abs())

    def backward(self, g):
        self.eh = self.eh + self.rounded
        self.bound()
        return super().backward(g)


FAR = {"spread 0.01 about 1000": lambda x: x * 0.01 + 1000.0, "spread 1 about -1e5": lambda x: x - 1e5,
       "1000 everywhere": lambda x: torch.full_like(x, 1000.0), "0.1 everywhere": lambda x: torch.full_like(x, 0.1),
       "one of many": lambda x: torch.cat([torch.full_like(x[:1], 1e4), x[1:]]), "as drawn": lambda x: x}


@pytest.mark.parametrize("how", list(FAR))
@pytest.mark.parametrize("kind", ["tiny", "molecules", "mixed", "large"])
@pytest.mark.parametrize("f,groups,xt", [(64, 8, "f32"), (24, 12, "f32"), (36, 6, "f32"), (33, 11, "f32"), (300, 1, "f32"),
                                         (64, 4, "bf16"), (35, 7, "bf16")])
def test_far_mean(how, kind, f, groups, xt):
    x, offsets, go, gamma, beta = make(kind, f, "f32", "f32", 40 + f, head=2, tail=3)
    x = FAR[how](x).to(DT[xt])
    off = torch.tensor(offsets, device="cuda")
    p = Far(x, offsets, groups, gamma, beta, "none")
    r = tfg.tfg_group_norm(x, off, groups, gamma, beta, EPS, "none", out_dtype=torch.float32)
    tfg.check_status(r.status)
    close(r.out[p.rows], p.out, p.out_tol, "out")
    close(r.mean, p.mean, p.mean_tol, "mean")
    close(r.rstd, p.rstd, p.rstd * p.rel, "rstd")
    grads = tfg.tfg_group_norm_backward(x, off, groups, gamma, beta, r.mean, r.rstd, go, "none")
    for got, (want, tol), name in zip((grads[0][p.rows], *grads[1:]), p.backward(go), ("grad_x", "grad_gamma", "grad_beta")):
        close(got, want, tol, name)


@pytest.mark.parametrize("value", [3.0, 1000.1, -7e4, 1e6, 3e28])
@pytest.mark.parametrize("sizes", [[3, 0, 7, 1, 13, 300], [5000, 1, 1111]])
@pytest.mark.parametrize("f,groups", [(64, 8), (33, 11), (24, 12)])
def test_equal_values_deviate_by_nothing(value, sizes, f, groups):
    """Whatever eps: no rounding of the mean is taken for a spread."""
    x = torch.full((sum(sizes), f), value, device="cuda")
    off = torch.tensor([0] + torch.tensor(sizes).cumsum(0).tolist(), device="cuda")
    beta = torch.linspace(-1, 1, f, device="cuda")
    for eps in (1e-5, 1e-30):
        r = tfg.tfg_group_norm(x, off, groups, None, beta, eps)
        assert torch.equal(r.out, beta.expand_as(x))
        held = torch.tensor([s > 0 for s in sizes], device="cuda")
        assert bool((r.mean[held] == x[0, 0]).all())
        close(r.rstd[held], torch.full_like(r.rstd[held], eps ** -0.5).double(), 8 * U * torch.full_like(r.rstd[held], eps ** -0.5), "rstd")


def test_infinities_and_the_range_of_squares():
    """An infinity makes its (graph, group) NaN, the first value or another; squares past fp32 a rstd of 0."""
    for kind in ("molecules", "large"):
        x, offsets, _, _, _ = make(kind, 32, "f32", "f32", 8)
        off = torch.tensor(offsets, device="cuda")
        clean = tfg.tfg_group_norm(x, off, 8).out
        a, b = next((a, b) for a, b in zip(offsets, offsets[1:]) if b - a > 3)
        mine = torch.zeros_like(x, dtype=torch.bool)
        mine[a:b, 8:12] = True
        for at in (a, a + 2):
            for bad in (float("inf"), -float("inf"), float("nan")):
                y = x.clone()
                y[at, 8] = bad
                r = tfg.tfg_group_norm(y, off, 8)
                assert bool(torch.isnan(r.out[mine]).all()) and torch.equal(r.out[~mine], clean[~mine])
            y = x.clone()
            y[a:b, 8:12] *= 1e30
            y[at, 8] = -3e38
            r = tfg.tfg_group_norm(y, off, 8)
            assert bool((r.out[mine] == 0).all()) and torch.equal(r.out[~mine], clean[~mine])
