"""Group norm with an activation, forward and backward, against plain 64-bit forms.

Tolerances are first-order error bounds, formed element by element in 64 bits, u = 2^-24.
No chain of fp32 additions here is longer than 512 (at most 220 rows a thread, 256 row lanes
and 1,024 / 32 channels a lane, never all three at once, then butterflies and one share in
32), so a sum of terms t is off by at most K sum |t| with K = 520 u.  Then, with A = mean |x| of the (graph,
group) and dm = K A the error of its mean,
  dr / r <= (K + 4 u) / 2 + (dm r)^2 / 2 + 2 u   (squares about m, a division, a root)
  eh = r dm + |h| (dr / r + 2 u),   ey = |gamma| eh + 2 u (|gamma h| + |beta|)
  out: 1.13 ey + 12 u (|y| + |act(y)|)   (largest slope 1.13; exp, erf and the quotient a few u)
  ed = |g| (ey + 12 u (1 + |y|))         (largest second derivative 0.8)
  s1: mean(|gamma| ed) + K mean |gamma d|, s2: mean(|gamma| (ed |h| + |d| eh)) + K mean |gamma d h|
  grad_x: r (|gamma| ed + es1 + |h| es2 + |s2| eh) + r (|gamma d| + |s1| + |h s2|) (dr / r + 6 u)
  grad_beta: sum ed + K sum |d|, grad_gamma: sum (ed |h| + |d| eh) + K sum |d h|
and half a step of bf16 (2^-8) where a result is stored so.  A ReLU's slope jumps at y = 0:
its gradients are compared on inputs whose |y| stays above ey.
"""
import math

import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import tfg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K = 520 * U
EPS = 1e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def act_of(y, name):
    """(act, slope) in 64 bits."""
    if name == "relu":
        return y.clamp(min=0), (y > 0).double()
    if name == "silu":
        p = torch.sigmoid(y)
        return y * p, p * (1 + y * (1 - p))
    if name == "gelu":
        p = torch.special.ndtr(y)
        return y * p, p + y * torch.exp(-y * y / 2) / math.sqrt(2 * math.pi)
    return y, torch.ones_like(y)


class Plain:
    """Values and error bounds of one batch (offsets: a list)."""

    def __init__(self, x, offsets, groups, gamma, beta, act, eps=EPS):
        n, f = x.shape
        self.n, self.f, self.k = n, f, groups
        self.offsets = offsets
        x = x.double()
        dev = x.device
        sizes = [b - a for a, b in zip(offsets, offsets[1:])]
        first, last = offsets[0], offsets[-1]
        self.rows = slice(first, last)
        self.graph = torch.repeat_interleave(torch.arange(len(sizes), device=dev), torch.tensor(sizes, device=dev))
        self.count = torch.tensor(sizes, device=dev).double()[:, None] * (f // groups)
        self.gamma = torch.ones(f, device=dev).double() if gamma is None else gamma.double()
        self.beta = torch.zeros(f, device=dev).double() if beta is None else beta.double()
        x = x[self.rows]
        self.mean = self.per_graph(x)
        c = x - self.spread(self.mean)
        self.rstd = (self.per_graph(c * c) + eps) ** -0.5
        self.rstd[self.count[:, 0] == 0] = 0
        dm = K * self.per_graph(x.abs())
        self.mean_tol = dm
        self.rel = (K + 4 * U) / 2 + (dm * self.rstd) ** 2 / 2 + 2 * U
        r = self.spread(self.rstd)
        self.h = c * r
        self.eh = r * self.spread(dm) + self.h.abs() * (self.spread(self.rel) + 2 * U)
        self.y = self.h * self.gamma + self.beta
        self.ey = self.gamma.abs() * self.eh + 2 * U * ((self.gamma * self.h).abs() + self.beta.abs())
        self.out, self.slope = act_of(self.y, act)
        self.out_tol = 1.13 * self.ey + 12 * U * (self.y.abs() + self.out.abs())

    def per_graph(self, v):
        """Means over the (graph, group) of v [rows, f]."""
        s = torch.zeros(len(self.count), self.k, dtype=torch.float64, device=v.device)
        s.index_add_(0, self.graph, v.reshape(v.shape[0], self.k, -1).sum(2))
        return s / self.count.clamp(min=1)

    def spread(self, s):
        return s[self.graph].repeat_interleave(self.f // self.k, 1)

    def backward(self, g):
        g = g.double()[self.rows]
        d = g * self.slope
        ed = g.abs() * (self.ey + 12 * U * (1 + self.y.abs()))
        ga, h = self.gamma, self.h
        s1, s2 = self.per_graph(ga * d), self.per_graph(ga * d * h)
        e1 = self.per_graph(ga.abs() * ed) + K * self.per_graph((ga * d).abs())
        e2 = self.per_graph(ga.abs() * (ed * h.abs() + d.abs() * self.eh)) + K * self.per_graph((ga * d * h).abs())
        r, s1, s2, e1, e2, rel = (self.spread(v) for v in (self.rstd, s1, s2, e1, e2, self.rel))
        gx = r * (ga * d - s1 - h * s2)
        gx_tol = r * (ga.abs() * ed + e1 + h.abs() * e2 + s2.abs() * self.eh) \
            + r * ((ga * d).abs() + s1.abs() + (h * s2).abs()) * (rel + 6 * U)
        gb, gb_tol = d.sum(0), ed.sum(0) + K * d.abs().sum(0)
        gg = (d * h).sum(0)
        gg_tol = (ed * h.abs() + d.abs() * self.eh).sum(0) + K * (d * h).abs().sum(0)
        return (gx, gx_tol), (gg, gg_tol), (gb, gb_tol)


def close(got, want, tol, what):
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {(off / tol.clamp(min=1e-300)).max():.3g} of the bound"


def sizes_of(kind, rng):
    return {"one": [1], "tiny": [0, 1, 2, 3, 0, 1, 5, 0], "rows": [1] * 300, "molecules": list(rng.integers(0, 201, 60)),
            "skew": [3, 0, 900, 1, 40, 2600, 7, 1, 130, 0], "large": [5000], "two_large": [2500, 3100], "mixed":
            [0, 4000, 0, 0, 12, 1500, 1, 1, 1, 2000, 0]}[kind]


def make(kind, f, xt, gt, seed, shift=1.0, head=0, tail=0):
    rng = np.random.default_rng(seed)
    sizes = sizes_of(kind, rng)
    offsets = np.concatenate([[head], head + np.cumsum(sizes)]).astype(np.int64)
    n = int(offsets[-1]) + tail
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, f, device="cuda", generator=g) * (0.5 + torch.rand(f, device="cuda", generator=g))
    x = (x + shift * torch.randn(f, device="cuda", generator=g)).to(DT[xt])
    go = torch.randn(n, f, device="cuda", generator=g).to(DT[gt])
    gamma = 1 + 0.3 * torch.randn(f, device="cuda", generator=g)
    beta = 0.3 * torch.randn(f, device="cuda", generator=g)
    return x, offsets.tolist(), go, gamma, beta


def run_and_check(x, offsets, groups, gamma, beta, act, go, ot, relu_margin=False):
    off = torch.tensor(offsets, device="cuda")
    n, f = x.shape
    p = Plain(x, offsets, groups, gamma, beta, act)
    out = torch.full((n, f), 7.0, device="cuda", dtype=DT[ot])
    r = tfg.tfg_group_norm(x, off, groups, gamma, beta, EPS, act, out=out)
    tfg.check_status(r.status)
    close(r.out[p.rows], p.out, p.out_tol, "out")
    close(r.mean, p.mean, p.mean_tol, "mean")
    close(r.rstd, p.rstd, p.rstd * p.rel, "rstd")
    rest = torch.cat([r.out[:offsets[0]], r.out[offsets[-1]:]])
    assert bool((rest == 7.0).all()), "rows outside the graphs are left as they were"
    grad_x = torch.full((n, f), 5.0, device="cuda", dtype=go.dtype)
    gx, gg, gb = tfg.tfg_group_norm_backward(x, off, groups, gamma, beta, r.mean, r.rstd, go, act, grad_x=grad_x)
    (wx, tx), (wg, tg), (wb, tb) = p.backward(go)
    if relu_margin:
        safe = p.y.abs() > 4 * p.ey
        assert float((~safe).double().mean()) < 1e-3
        if not bool(safe.all()):
            return
    close(gx[p.rows], wx, tx, "grad_x")
    close(gg, wg, tg, "grad_gamma")
    close(gb, wb, tb, "grad_beta")
    assert bool((torch.cat([gx[:offsets[0]], gx[offsets[-1]:]]) == 5.0).all())
    again = tfg.tfg_group_norm_backward(x, off, groups, gamma, beta, r.mean, r.rstd, go, act)
    assert torch.equal(again[0][p.rows], gx[p.rows]) and torch.equal(again[1], gg) and torch.equal(again[2], gb)
    alone = tfg.tfg_group_norm_backward(x, off, groups, gamma, beta, r.mean, r.rstd, go, act, want_weight_grads=False)
    assert alone[1] is None and torch.equal(alone[0][p.rows], gx[p.rows])
    bare = tfg.tfg_group_norm(x, off, groups, gamma, beta, EPS, act, out_dtype=DT[ot], want_stats=False)
    assert bare.mean is None and torch.equal(bare.out[p.rows], r.out[p.rows])


LAYOUTS = [(1, 1), (3, 1), (4, 4), (6, 2), (8, 8), (24, 3), (64, 8), (100, 25), (123, 41), (128, 32), (256, 2), (260, 1)]


@pytest.mark.parametrize("kind", ["one", "tiny", "rows", "molecules", "skew", "large", "two_large", "mixed"])
@pytest.mark.parametrize("f,groups", LAYOUTS)
def test_layouts_and_sizes(kind, f, groups):
    xt, gt, act = [("f32", "f32", "silu"), ("bf16", "bf16", "gelu"), ("bf16", "f32", "none")][(f + len(kind)) % 3]
    x, offsets, go, gamma, beta = make(kind, f, xt, gt, f * 7 + groups)
    run_and_check(x, offsets, groups, gamma, beta, act, go, gt)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("kind,f,groups", [("skew", 64, 16), ("molecules", 40, 5), ("mixed", 33, 11)])
def test_types_and_activations(xt, gt, act, kind, f, groups):
    x, offsets, go, gamma, beta = make(kind, f, xt, gt, 11)
    run_and_check(x, offsets, groups, gamma, beta, act, go, gt)


@pytest.mark.parametrize("kind", ["molecules", "large"])
def test_relu(kind):
    x, offsets, go, gamma, beta = make(kind, 32, "f32", "f32", 5)
    # values on a grid wide against the bound: no y near 0
    x = torch.round(x * 4) / 4 + 0.01
    run_and_check(x, offsets, 8, gamma, beta, "relu", go, "f32", relu_margin=True)


def test_relu_backward_at_the_sign_of_y():
    """The slope is 1 where the forward gave a positive value and 0 where it gave 0."""
    x, offsets, go, _, _ = make("skew", 16, "f32", "f32", 6)
    off = torch.tensor(offsets, device="cuda")
    r = tfg.tfg_group_norm(x, off, 4, activation="relu")
    _, _, gb = tfg.tfg_group_norm_backward(x, off, 4, None, None, r.mean, r.rstd, go, "relu")
    d = go.double() * (r.out > 0)
    close(gb, d.sum(0), K * d.abs().sum(0), "grad_beta")


@pytest.mark.parametrize("f,groups", [(1024, 1), (1000, 1), (1023, 1), (2046, 2), (2048, 2), (4096, 4), (3000, 3), (1536, 512)])
@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_wide_groups(f, groups, xt):
    """Up to 1,024 channels a group, with and without whole vectors."""
    for kind in ("tiny", "molecules"):
        x, offsets, go, gamma, beta = make(kind, f, xt, xt, f)
        run_and_check(x, offsets, groups, gamma, beta, "silu", go, xt)


@pytest.mark.parametrize("head,tail", [(0, 5), (3, 0), (17, 900)])
@pytest.mark.parametrize("kind", ["molecules", "mixed"])
def test_rows_outside_the_graphs(head, tail, kind):
    x, offsets, go, gamma, beta = make(kind, 48, "f32", "f32", 3, head=head, tail=tail)
    x[:head], x[offsets[-1]:] = math.nan, math.inf
    go[:head], go[offsets[-1]:] = math.inf, math.nan
    run_and_check(x, offsets, 12, gamma, beta, "gelu", go, "f32")


@pytest.mark.parametrize("gamma_on,beta_on", [(False, False), (True, False), (False, True)])
def test_without_weights(gamma_on, beta_on):
    x, offsets, go, gamma, beta = make("skew", 72, "f32", "f32", 9)
    run_and_check(x, offsets, 9, gamma if gamma_on else None, beta if beta_on else None, "silu", go, "f32")


@pytest.mark.parametrize("kind", ["molecules", "large"])
def test_far_mean_constant_and_small_values(kind):
    for make_x in (lambda x: x * 0.01 + 1000.0, lambda x: x * 0 + 3.0, lambda x: x * 1e-6, lambda x: x * 1e6,
                   lambda x: torch.cat([torch.full_like(x[:1], 1e4), x[1:]])):
        x, offsets, go, gamma, beta = make(kind, 64, "f32", "f32", 4)
        run_and_check(make_x(x), offsets, 8, gamma, beta, "none", go, "f32")


def test_misaligned():
    for f, groups in ((64, 8), (12, 3)):
        for dt in ("f32", "bf16"):
            x, offsets, go, gamma, beta = make("skew", f, dt, dt, 8)
            n = x.shape[0]
            buf = torch.empty(n * f + 1, device="cuda", dtype=DT[dt])
            buf[1:] = x.view(-1)
            run_and_check(buf[1:].view(n, f), offsets, groups, gamma, beta, "silu", go, dt)


def test_not_finite_values_stay_in_their_graph_and_group():
    x, offsets, go, gamma, beta = make("mixed", 32, "f32", "f32", 2)
    off = torch.tensor(offsets, device="cuda")
    clean = tfg.tfg_group_norm(x, off, 8, gamma, beta)
    row = {1: 100, 4: offsets[4] + 2}
    for graph, at in row.items():
        y = x.clone()
        y[at, 9] = math.inf if graph == 1 else math.nan
        r = tfg.tfg_group_norm(y, off, 8, gamma, beta)
        mine = torch.zeros_like(x, dtype=torch.bool)
        mine[offsets[graph]:offsets[graph + 1], 8:12] = True
        assert torch.equal(r.out[~mine], clean.out[~mine])
        assert bool((~torch.isfinite(r.out[mine])).any())
        gx, _, _ = tfg.tfg_group_norm_backward(y, off, 8, gamma, beta, r.mean, r.rstd, go)
        good, _, _ = tfg.tfg_group_norm_backward(x, off, 8, gamma, beta, clean.mean, clean.rstd, go)
        assert torch.equal(gx[~mine], good[~mine])


def test_bad_offsets_are_reported():
    x = torch.randn(500, 16, device="cuda")
    for bad in ([0, 600], [0, 300, 200, 500], [-1, 500], [0, 10, 2**40]):
        r = tfg.tfg_group_norm(x, torch.tensor(bad, device="cuda"), 4)
        assert int(r.status) == tfg.TFG_ERR_INDEX_RANGE, bad
        tfg.tfg_group_norm_backward(x, torch.tensor(bad, device="cuda"), 4, None, None, r.mean, r.rstd, x.clone())
    torch.cuda.synchronize()
    r = tfg.tfg_group_norm(x, torch.tensor([0, 500], device="cuda"), 4)
    tfg.check_status(r.status)


def test_no_graphs_and_no_rows():
    x = torch.randn(10, 8, device="cuda")
    out = torch.full_like(x, 3.0)
    r = tfg.tfg_group_norm(x, torch.tensor([0], device="cuda"), 2, out=out)
    tfg.check_status(r.status)
    assert bool((r.out == 3.0).all()) and r.mean.shape == (0, 2)
    _, gg, gb = tfg.tfg_group_norm_backward(x, torch.tensor([4], device="cuda"), 2, None, None, r.mean, r.rstd, x.clone())
    assert bool((gg == 0).all()) and bool((gb == 0).all())
    none = x[:0]
    r = tfg.tfg_group_norm(none, torch.zeros(4, dtype=torch.int64, device="cuda"), 2)
    tfg.check_status(r.status)
    assert bool((r.mean == 0).all()) and bool((r.rstd == 0).all())
    _, gg, gb = tfg.tfg_group_norm_backward(none, torch.zeros(4, dtype=torch.int64, device="cuda"), 2, None, None, r.mean,
                                            r.rstd, none.clone())
    assert bool((gg == 0).all()) and bool((gb == 0).all())
    _, gg, gb = tfg.tfg_group_norm_backward(x, torch.full((4,), 5, device="cuda"), 2, None, None, r.mean, r.rstd, x.clone())
    assert bool((gg == 0).all()) and bool((gb == 0).all())


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("kind", ["molecules", "two_large"])
def test_gradient_against_differences(act, kind):
    """<grad, v> against a central difference of the 64-bit forward along random v; the
    difference's own error is its third derivative's, h^2 / 6 of a value of order 1 (at
    most 100 times the sum's scale for these inputs): h = 1e-4 leaves 1e-6 of it."""
    x, offsets, go, gamma, beta = make(kind, 24, "f32", "f32", 21)
    off = torch.tensor(offsets, device="cuda")
    r = tfg.tfg_group_norm(x, off, 6, gamma, beta, EPS, act)
    grads = tfg.tfg_group_norm_backward(x, off, 6, gamma, beta, r.mean, r.rstd, go, act)
    bounds = [t for _, t in Plain(x, offsets, 6, gamma, beta, act).backward(go)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = 1e-4
    for i, (at, grad) in enumerate(zip((x, gamma, beta), grads)):
        v = torch.randn(at.shape, device="cuda", dtype=torch.float64, generator=gen)
        ends = []
        for sign in (1, -1):
            moved = [t.double() + (sign * h * v if j == i else 0) for j, t in enumerate((x, gamma, beta))]
            ends.append(float((Plain(moved[0], offsets, 6, moved[1], moved[2], act).out * go.double()).sum()))
        got = float((grad.double() * v).sum())
        scale = float((grad.double() * v).abs().sum())
        assert abs(got - (ends[0] - ends[1]) / (2 * h)) <= float((bounds[i] * v.abs()).sum()) + 1e-6 * scale


def test_captured_and_on_another_stream():
    x, offsets, go, gamma, beta = make("mixed", 64, "f32", "f32", 1)
    off = torch.tensor(offsets, device="cuda")
    n, f = x.shape
    need = max(tfg.tfg_group_norm_workspace_size(n, len(offsets) - 1, f, 8),
               tfg.tfg_group_norm_backward_workspace_size(n, len(offsets) - 1, f, 8))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        r = tfg.tfg_group_norm(x, off, 8, gamma, beta, EPS, "silu", workspace=ws)
        return r, tfg.tfg_group_norm_backward(x, off, 8, gamma, beta, r.mean, r.rstd, go, "silu", workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, grads = step()
    for kind, seed in (("mixed", 31), ("mixed", 32)):
        y, _, go2, _, _ = make(kind, f, "f32", "f32", seed)
        x.copy_(y)
        go.copy_(go2)
        # the offsets are data: the same batch shape with other graph sizes
        new = sorted(np.random.default_rng(seed).integers(0, n + 1, len(offsets) - 2).tolist())
        off.copy_(torch.tensor([0] + new + [n], device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        p = Plain(x, off.tolist(), 8, gamma, beta, "silu")
        tfg.check_status(r.status)
        close(r.out, p.out, p.out_tol, "out")
        for got, (want, tol), name in zip(grads, p.backward(go), ("grad_x", "grad_gamma", "grad_beta")):
            close(got, want, tol, name)


def test_more_than_2_32_elements():
    n, f, groups = (1 << 25) + 77, 136, 17
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(n, f, device="cuda", generator=g, dtype=torch.bfloat16)
    edges = [0, 1, 300, n - 5000, n - 4990, n - 2, n]
    off = torch.tensor(edges, device="cuda")
    r = tfg.tfg_group_norm(x, off, groups, activation="silu")
    tfg.check_status(r.status)
    gx, gg, gb = tfg.tfg_group_norm_backward(x, off, groups, None, None, r.mean, r.rstd, r.out, "silu")
    small = edges[3:]                      # the last graphs, compared as a batch of their own
    at = small[0]
    p = Plain(x[at:], [e - at for e in small], groups, None, None, "silu")
    close(r.out[at:], p.out, p.out_tol, "out")
    close(r.mean[3:], p.mean, p.mean_tol, "mean")
    (wx, tx), _, _ = p.backward(r.out[at:])
    close(gx[at:], wx, tx, "grad_x")
    # the large graph: statistics of 5.7e8 normal values a group (five sigma of the sample), and
    # its rows from the reported statistics
    m = (edges[3] - edges[2]) * (f // groups)
    assert float(r.mean[2].abs().max()) < 5 / math.sqrt(m) + K
    assert float((r.rstd[2] - 1).abs().max()) < 5 / math.sqrt(m) + 2.0 ** -7 + K + EPS
    rows = torch.tensor([300, 301, n // 2, edges[3] - 1], device="cuda")
    y = (x[rows].double() - r.mean[2].double().repeat_interleave(8)) * r.rstd[2].double().repeat_interleave(8)
    want = y * torch.sigmoid(y)
    close(r.out[rows], want, 20 * U * (1 + y.abs()), "rows of the large graph")


def test_binding_refuses():
    x, off = torch.randn(10, 8, device="cuda"), torch.tensor([0, 10], device="cuda")
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x.t(), off, 2)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x, off.int(), 2)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x, off, 2, gamma=torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x, off, 2, activation="tanh")
    with pytest.raises(tfg.TfgError):
        tfg.tfg_group_norm(x, off, 3)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_group_norm(x, off, 2, out=x)                              # in place
    r = tfg.tfg_group_norm(x, off, 2)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm_backward(x, off, 2, None, None, r.mean, r.rstd, x[:5])
    with pytest.raises(ValueError):
        tfg.tfg_group_norm_backward(x, off, 2, None, None, r.mean[:, :1].contiguous(), r.rstd, x.clone())
