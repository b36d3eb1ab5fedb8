"""Calls that the documentation of the embedding, group-norm and clipping entry points allows
and that ordinary batches do not make: very many graphs, one graph in very many shares,
status words of long lists, weights off the vector boundary, calls from several threads,
and the bounds-checked build."""
import os
import threading

import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import build, tfg
from test_gpu_group_norm import EPS, Plain, close, make, run_and_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()


def features(n, f, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, f, device="cuda", generator=g) + torch.randn(f, device="cuda", generator=g)
    return x.to(dtype), torch.randn(n, f, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("graphs,most,f,groups", [(9000, 4, 16, 2), (300_000, 2, 8, 2), (20_000, 30, 33, 11)])
def test_very_many_graphs(graphs, most, f, groups):
    sizes = np.random.default_rng(graphs).integers(0, most + 1, graphs)
    sizes[graphs // 3] = 700                                  # one that no team holds
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    x, go = features(int(offsets[-1]), f, 1)
    gamma = torch.linspace(0.5, 1.5, f, device="cuda")
    run_and_check(x, offsets.tolist(), groups, gamma, None, "none", go, "f32")
    bad = torch.tensor(offsets, device="cuda")
    bad[graphs // 2] = bad[-1] + 5
    r = tfg.tfg_group_norm(x, bad, groups)
    assert int(r.status) == tfg.TFG_ERR_INDEX_RANGE


@pytest.mark.parametrize("sizes", [[150_000], [5, 0, 140_000, 3, 9_999], [70_001, 70_002]])
@pytest.mark.parametrize("f,groups,dt", [(64, 64, "bf16"), (96, 32, "f32"), (40, 1, "f32"), (24, 8, "bf16")])
def test_graphs_of_very_many_shares(sizes, f, groups, dt):
    """Partial statistics joined by a kernel of their own, or by every team for itself."""
    offsets = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    x, go = features(offsets[-1], f, 2, torch.bfloat16 if dt == "bf16" else torch.float32)
    run_and_check(x, offsets, groups, None, torch.linspace(-0.2, 0.2, f, device="cuda"), "silu", go, dt)


def test_weights_off_the_vector_boundary():
    x, offsets, go, gamma, beta = make("skew", 32, "f32", "f32", 3)
    buf = torch.empty(65, device="cuda")
    g, b = buf[1:33], buf[33:65]
    g.copy_(gamma)
    b.copy_(beta)
    run_and_check(x, offsets, 8, g, b, "gelu", go, "f32")


@pytest.mark.parametrize("n", [8192, 8193, 50_000])
def test_status_of_long_lists(n):
    table = torch.randn(100, 12, device="cuda")
    ids = torch.randint(0, 100, (n,), device="cuda")
    for at in (None, 0, n // 2, n - 1):
        now = ids.clone()
        if at is not None:
            now[at] = 100
        out, status = tfg.tfg_embedding_lookup(table, now)
        groups = tfg.tfg_group_ids(now, 100)
        want = 0 if at is None else tfg.TFG_ERR_INDEX_RANGE
        assert int(status) == want and int(groups.status) == want
        if at is not None:
            assert bool((out[at] == 0).all()) and int(groups.rowptr[100]) == n - 1


def test_wide_rows_and_many_column_tiles():
    for f, dt in ((5000, torch.bfloat16), (40_003, torch.float32)):
        table = torch.randn(7, f, device="cuda").to(dt)
        ids = torch.randint(0, 7, (400,), device="cuda")
        out, _ = tfg.tfg_embedding_lookup(table, ids, 1.0)
        assert torch.equal(out, table[ids])
        grad = torch.randn(400, f, device="cuda").to(dt)
        got = tfg.tfg_embedding_backward(tfg.tfg_group_ids(ids, 7), grad)
        want = torch.zeros(7, f, dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double())
        size = torch.zeros(7, f, dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double().abs())
        assert bool(((got.double() - want).abs() <= 404 * 2.0 ** -24 * size).all())


def test_from_several_threads():
    """Calls of different sizes from threads of their own, each on its own stream."""
    jobs = [make(kind, f, "f32", "f32", i) for i, (kind, f) in enumerate([("molecules", 64), ("large", 128), ("tiny", 24)])]
    alone = []
    for x, offsets, go, gamma, beta in jobs:
        off = torch.tensor(offsets, device="cuda")
        r = tfg.tfg_group_norm(x, off, 8, gamma, beta, EPS, "silu")
        alone.append((off, r, tfg.tfg_group_norm_backward(x, off, 8, gamma, beta, r.mean, r.rstd, go, "silu")))
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        try:
            x, _, go, gamma, beta = jobs[i]
            off, want, want_back = alone[i]
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    r = tfg.tfg_group_norm(x, off, 8, gamma, beta, EPS, "silu")
                    back = tfg.tfg_group_norm_backward(x, off, 8, gamma, beta, r.mean, r.rstd, go, "silu")
                torch.cuda.current_stream().synchronize()
                if not (torch.equal(r.out, want.out) and all(torch.equal(a, b) for a, b in zip(back, want_back))):
                    wrong.append(i)
        except Exception as e:                               # seen by the main thread
            wrong.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong


def test_norm_of_one_value_and_of_equal_values():
    x = torch.tensor([[3.0], [5.0], [5.0]], device="cuda")
    r = tfg.tfg_group_norm(x, torch.tensor([0, 1, 3], device="cuda"), 1, beta=torch.tensor([0.25], device="cuda"))
    assert r.out.flatten().tolist() == [0.25, 0.25, 0.25]
    gx, gg, gb = tfg.tfg_group_norm_backward(x, torch.tensor([0, 1, 3], device="cuda"), 1, None, None, r.mean, r.rstd,
                                             torch.ones_like(x))
    assert gx.flatten().tolist() == [0.0, 0.0, 0.0] and float(gg) == 0.0 and float(gb) == 3.0


def test_bounds_checked_build():
    path = os.path.join(build.OBJ_DIR, "libtfg_checked.so")
    newest = max(os.path.getmtime(p) for p in build._deps())
    if not os.path.exists(path) or os.path.getmtime(path) < newest:
        build.build_library(defines=("TFG_CHECK_BOUNDS=1",), lib_path=path)
    x, offsets, go, gamma, beta = make("mixed", 32, "f32", "f32", 7)
    off = torch.tensor(offsets, device="cuda")
    ids = torch.randint(0, 30, (5000,), device="cuda")
    table = torch.randn(30, 16, device="cuda")

    def step():
        r = tfg.tfg_group_norm(x, off, 8, gamma, beta, EPS, "silu")
        back = tfg.tfg_group_norm_backward(x, off, 8, gamma, beta, r.mean, r.rstd, go, "silu")
        out, _ = tfg.tfg_embedding_lookup(table, ids, 3.0)
        grad = tfg.tfg_embedding_backward(tfg.tfg_group_ids(ids, 30), out)
        clipped, norm = tfg.tfg_clip_by_global_norm([grad, back[1]], 0.5)
        torch.cuda.synchronize()
        return [r.out, *back, out, grad, norm, *clipped]

    want = step()
    tfg.use_library(path)
    try:
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
        # A table of ten rows at the end of an allocation, and a call that says twenty: refused,
        # nothing launched.  Every id is 0, and ids and out lie in the same allocation, so that
        # even a launch would stay within it.
        torch.cuda.empty_cache()
        buf = torch.zeros((32 << 20) // 4, device="cuda")
        seg = [s for s in torch.cuda.memory_snapshot()
               if s["address"] <= buf.data_ptr() < s["address"] + s["total_size"]]
        if not seg or seg[0]["address"] + seg[0]["total_size"] != buf.data_ptr() + buf.numel() * 4:
            pytest.skip("the caching allocator did not give the buffer a segment of its own")
        at = buf.data_ptr()
        rc = tfg.lib().tfg_embedding_lookup(at, 5000, buf[-160:].data_ptr(), 0, 20, 16, 1.0, -1, at + (1 << 20), 0,
                                            at + (8 << 20), None)
        msg = tfg.tfg_last_error()
        assert rc == tfg.TFG_ERR_INDEX_RANGE and "table must hold" in msg, (rc, msg)
    finally:
        tfg.use_library(build.LIB_PATH)


@pytest.mark.parametrize("n,f", [(127, 128), (128, 128), (129, 128), (255, 128), (256, 128), (257, 128), (2047, 16), (2048, 16),
                                 (2049, 16), (1024, 24), (1025, 24)])
@pytest.mark.parametrize("rows", [1, 3, 40_000])
def test_gradient_around_one_cta(n, f, rows):
    """Lists that one CTA reduces, and those one longer, whose rows may cross CTAs."""
    ids = torch.randint(0, rows, (n,), device="cuda")
    ids[: n // 2] = rows // 2                                 # one id with half of the positions
    grad = torch.randn(n, f, device="cuda")
    got = tfg.tfg_embedding_backward(tfg.tfg_group_ids(ids, rows), grad, 0.5)
    want = torch.zeros(rows, f, dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double()) * 0.5
    size = torch.zeros(rows, f, dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double().abs()) * 0.5
    assert bool(((got.double() - want).abs() <= (n + 4) * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("f,groups,dt", [(35, 7, "f32"), (35, 7, "bf16"), (400, 25, "f32"), (75, 25, "f32"), (1023, 3, "f32")])
def test_graphs_of_a_few_rows(f, groups, dt):
    """Small unequal graphs: some fit a team only by the room that it has anyway, some do not."""
    sizes = np.random.default_rng(f).geometric(1 / 3, 900) - 1
    sizes[::100] = [63, 64, 65, 66, 130, 12, 13, 14, 200]
    offsets = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    x, go = features(offsets[-1], f, 4, torch.bfloat16 if dt == "bf16" else torch.float32)
    run_and_check(x, offsets, groups, torch.linspace(0.5, 1.5, f, device="cuda"), None, "silu", go, dt)
