"""A batch of one large graph and very many small ones: the work on the large graph grows with
its rows, not with the square of them."""
import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_group_norm import EPS, Plain, close

pytestmark = pytest.mark.gpu
F, GROUPS = 128, 32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def batch(sizes):
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    g = torch.Generator(device="cuda").manual_seed(int(offsets[-1]))
    x = torch.randn(int(offsets[-1]), F, device="cuda", generator=g) + torch.randn(F, device="cuda", generator=g)
    return x, torch.tensor(offsets, device="cuda"), torch.randn_like(x)


def best_ms(call, times=5):
    call()
    ms = []
    for _ in range(times):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        ms.append(a.elapsed_time(b))
    return min(ms)


def calls(x, off, go):
    r = tfg.tfg_group_norm(x, off, GROUPS, eps=EPS, activation="silu")
    return (lambda: tfg.tfg_group_norm(x, off, GROUPS, eps=EPS, activation="silu"),
            lambda: tfg.tfg_group_norm_backward(x, off, GROUPS, None, None, r.mean, r.rstd, go, "silu"))


@pytest.mark.parametrize("large,small", [(500_000, 30_000), (240_000, 4095), (900_000, 50_000)])
def test_time_follows_the_rows(large, small):
    """Against the same number of rows in graphs of 100, whose work is the rows': the large
    graph reads its rows twice and its small neighbours are graphs of a few rows, so up to
    four times as long is granted; a join of all pieces in every piece took ten times as long and more."""
    rng = np.random.default_rng(small)
    sizes = rng.integers(1, 6, small + 1)
    sizes[small // 2] = large
    skewed = calls(*batch(sizes))
    even = calls(*batch([100] * (int(sizes.sum()) // 100)))
    for name, a, b in zip(("forward", "backward"), skewed, even):
        got, base = best_ms(a), best_ms(b)
        print(f"{name}: {got:.3f} ms against {base:.3f} ms in even graphs")
        assert got <= 4 * base, f"{name}: {got:.3f} ms against {base:.3f} ms"


@pytest.mark.parametrize("large,small", [([60_000], 3000), ([20_000, 1, 30_000], 5000), ([9000] * 7, 700)])
def test_values(large, small):
    rng = np.random.default_rng(small)
    sizes = rng.integers(0, 6, small)
    at = np.sort(rng.choice(small, len(large), replace=False))
    sizes[at] = large
    x, off, go = batch(sizes)
    p = Plain(x, off.tolist(), GROUPS, None, None, "silu")
    r = tfg.tfg_group_norm(x, off, GROUPS, eps=EPS, activation="silu")
    tfg.check_status(r.status)
    close(r.out, p.out, p.out_tol, "out")
    close(r.mean, p.mean, p.mean_tol, "mean")
    close(r.rstd, p.rstd, p.rstd * p.rel, "rstd")
    grads = tfg.tfg_group_norm_backward(x, off, GROUPS, None, None, r.mean, r.rstd, go, "silu")
    for got, (want, tol), name in zip(grads, p.backward(go), ("grad_x", "grad_gamma", "grad_beta")):
        close(got, want, tol, name)
