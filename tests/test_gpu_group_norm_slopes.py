"""Backward of the group norm's activations: the ReLU with every gradient compared, and values
where exponentials leave the range of fp32.

Bounds: those of test_gpu_group_norm.  A ReLU's slope jumps at y = 0: where |y| is within the
forward's error of 0 the gradient that comes in is 0, so that either slope gives the same."""
import math

import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_group_norm import DT, EPS, U, Plain, close, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def both(x, offsets, groups, gamma, beta, act, go):
    off = torch.tensor(offsets, device="cuda")
    r = tfg.tfg_group_norm(x, off, groups, gamma, beta, EPS, act, out_dtype=go.dtype)
    tfg.check_status(r.status)
    return r, tfg.tfg_group_norm_backward(x, off, groups, gamma, beta, r.mean, r.rstd, go, act)


def compare(p, r, grads, go):
    close(r.out[p.rows], p.out, p.out_tol, "out")
    for got, (want, tol), name in zip((grads[0][p.rows], *grads[1:]), p.backward(go), ("grad_x", "grad_gamma", "grad_beta")):
        close(got, want, tol, name)


@pytest.mark.parametrize("xt", ["f32", "bf16"])
@pytest.mark.parametrize("gt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["one", "tiny", "rows", "molecules", "skew", "large", "mixed"])
@pytest.mark.parametrize("f,groups", [(32, 8), (33, 11), (24, 12), (128, 2), (300, 1)])
def test_relu(kind, f, groups, xt, gt):
    x, offsets, go, gamma, beta = make(kind, f, xt, gt, 17)
    p = Plain(x, offsets, groups, gamma, beta, "relu")
    unsafe = p.y.abs() <= 2 * p.ey
    assert float(unsafe.double().mean()) < 0.01
    go[p.rows][unsafe] = 0
    r, grads = both(x, offsets, groups, gamma, beta, "relu", go)
    compare(p, r, grads, go)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("kind", ["molecules", "large"])
@pytest.mark.parametrize("xt", ["f32", "bf16"])
def test_far_from_zero(act, kind, xt):
    """y from -300 to 300, past the ends of e^y and e^(-y^2 / 2); and 1e30, where all is slope 0 or 1."""
    x, offsets, go, gamma, beta = make(kind, 32, xt, "f32", 23)
    for factor in (100.0, 1e30):
        p = Plain(x, offsets, 8, gamma * factor, beta, act)
        assert float(p.y.max()) > 2 * factor and float(p.y.min()) < -2 * factor
        safe = p.y.abs() > 60 if factor == 100.0 else p.y.abs() > 1e26    # the slopes in between: by the other tests
        g = torch.where(safe, go[p.rows].double(), 0.0).to(go.dtype)
        full = torch.zeros_like(go)
        full[p.rows] = g
        r, grads = both(x, offsets, 8, gamma * factor, beta, act, full)
        assert bool(torch.isfinite(r.out[p.rows]).all()) and all(bool(torch.isfinite(t).all()) for t in grads[1:])
        close(r.out[p.rows][safe], p.out[safe], p.out_tol[safe], "out")
        # slopes of 0 and 1 within |y| e^-60: the gradients without an activation where y > 0
        want = Plain(x, offsets, 8, gamma * factor, beta, "none")
        pass_on = full.clone()
        pass_on[p.rows] = torch.where(p.y > 0, full[p.rows].double(), 0.0).to(full.dtype)
        # the gradient comes in exactly, not off by the slope's error: what is left are sums
        want.ey, want.y = torch.zeros_like(want.ey), torch.zeros_like(want.y)
        for got, (w, tol), name in zip((grads[0][p.rows], *grads[1:]), want.backward(pass_on), ("grad_x", "grad_gamma", "grad_beta")):
            close(got, w, tol + 12 * U * w.abs(), name)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("kind", ["molecules", "mixed"])
def test_not_finite_values_with_every_activation(act, kind):
    x, offsets, go, gamma, beta = make(kind, 32, "f32", "f32", 2)
    clean, good = both(x, offsets, 8, gamma, beta, act, go)
    a, b = [(a, b) for a, b in zip(offsets, offsets[1:]) if b - a > 5][1]
    mine = torch.zeros_like(x, dtype=torch.bool)
    mine[a:b, 8:12] = True
    for bad in (math.inf, -math.inf, math.nan):
        y = x.clone()
        y[a + 4, 9] = bad
        r, grads = both(y, offsets, 8, gamma, beta, act, go)
        assert torch.equal(r.out[~mine], clean.out[~mine]) and torch.equal(grads[0][~mine], good[0][~mine])
        assert bool(torch.isnan(r.out[mine]).all()) and bool(torch.isnan(grads[0][mine]).all())
        for got, want in zip(grads[1:], good[1:]):
            assert torch.equal(got[:8], want[:8]) and torch.equal(got[12:], want[12:])
        assert bool(torch.isnan(grads[1][8:12]).all())
        assert act == "none" or bool(torch.isnan(grads[2][8:12]).all())  # without one, grad_beta is a sum of grad_out
        g = go.clone()
        g[a + 4, 9] = bad
        _, grads = both(x, offsets, 8, gamma, beta, act, g)
        assert torch.equal(grads[0][~mine], good[0][~mine])
        assert torch.equal(grads[2][:9], good[2][:9]) and torch.equal(grads[2][10:], good[2][10:])
