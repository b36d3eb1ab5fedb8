"""Embedding, GCN aggregation, group norm with its activation, pooling and their backwards,
and clipping, run together as a training step of a small graph classifier does, against
the same step in 64 bits under autograd on the CPU.

The step:  x = scale E[ids];  h = Ahat x;  y = silu(group_norm(h));  p = mean pool of y per
graph;  loss = <w, p>.  Every operator's own test bounds its error; here the gradients of
the whole chain are held to 2e-5 of their 2-norm: a chain of six operators, each within
some 1e-6 (fp32 sums of up to 500 terms, u = 6e-8, in blocks), whose norms do not shrink
an error by more than the condition of the group norm (h has a spread of about 1 here).
"""
import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import graphgen as gg
from paper_2101_11552_gb300 import tfg
from _helpers import dev

pytestmark = pytest.mark.gpu
KINDS, F, GROUPS, GRAPHS = 30, 48, 12, 37
SCALE = float(np.float32(np.sqrt(F)))
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def batch(seed):
    """Graphs of 2 to 120 nodes, batched on the device; ids of the nodes, some of them padding."""
    rng = np.random.default_rng(seed)
    sizes = rng.integers(2, 121, GRAPHS)
    parts = [gg.with_self_loops(gg.symmetrise(gg.er_pairs(int(s), int(s) - 1, rng)), int(s)) for s in sizes]
    stacked = np.ascontiguousarray(np.concatenate(parts, axis=1))
    counts = np.array([p.shape[1] for p in parts], np.int64)
    b = tfg.tfg_batch_graphs(dev(sizes.astype(np.int64)), dev(counts), dev(stacked), int(sizes.sum()))
    tfg.check_status(b.status)
    ids = rng.integers(0, KINDS, int(sizes.sum()))
    ids[rng.random(len(ids)) < 0.05] = -1
    return b, dev(ids)


def step(b, csr, src, dinv, ids, table, gamma, beta, w, clip):
    """One training step on the device: (pooled, gradients clipped, norm before)."""
    x, st = tfg.tfg_embedding_lookup(table, ids, SCALE, padding_id=-1)
    h = tfg.tfg_gcn_aggregate_sum(csr.rowptr, csr.col, dinv, x)
    y = tfg.tfg_group_norm(h, b.node_offsets, GROUPS, gamma, beta, EPS, "silu")
    pooled, _ = tfg.tfg_segment_pool(y.out, b.batch, GRAPHS, "mean")
    counts = (b.node_offsets[1:] - b.node_offsets[:-1]).float()
    gy = (w / counts[:, None])[b.batch]                       # dloss/dy of the mean pool
    gh, g_gamma, g_beta = tfg.tfg_group_norm_backward(h, b.node_offsets, GROUPS, gamma, beta, y.mean, y.rstd, gy, "silu")
    gx = tfg.tfg_gcn_aggregate_backward(src, dinv, gh)
    groups = tfg.tfg_group_ids(ids, KINDS, padding_id=-1)
    g_table = tfg.tfg_embedding_backward(groups, gx, SCALE)
    grads, norm = tfg.tfg_clip_by_global_norm([g_table, g_gamma, g_beta], clip)
    return pooled, grads, norm, [st, y.status, groups.status]


def plain(b, dinv_edges, ids, table, gamma, beta, w, clip):
    """The same in 64 bits on the CPU, gradients by autograd."""
    src, dst, weight = dinv_edges
    n = ids.numel()
    t, ga, be = (v.double().cpu().requires_grad_() for v in (table, gamma, beta))
    here = ids.cpu() != -1
    x = torch.zeros(n, F, dtype=torch.float64).index_add(0, torch.nonzero(here).flatten(), t[ids.cpu()[here]] * SCALE)
    h = torch.zeros(n, F, dtype=torch.float64).index_add(0, dst, x[src] * weight[:, None])
    out = []
    offs = b.node_offsets.tolist()
    for a, e in zip(offs, offs[1:]):
        v = h[a:e].reshape(e - a, GROUPS, -1)
        m = v.mean((0, 2), keepdim=True)
        v = (v - m) / torch.sqrt(((v - m) ** 2).mean((0, 2), keepdim=True) + EPS)
        y = v.reshape(e - a, F) * ga + be
        out.append((y * torch.sigmoid(y)).mean(0))
    pooled = torch.stack(out)
    (pooled * w.double().cpu()).sum().backward()
    grads = [t.grad, ga.grad, be.grad]
    norm = float(torch.sqrt(sum((g ** 2).sum() for g in grads)))
    return pooled.detach(), [g * (clip / max(norm, clip)) for g in grads], norm


def gcn_weights(b, n):
    ei = b.edge_index.cpu()
    deg = torch.zeros(n, dtype=torch.float64).index_add(0, ei[1], torch.ones(ei.shape[1], dtype=torch.float64))
    return ei[0], ei[1], (deg[ei[0]] * deg[ei[1]]) ** -0.5


@pytest.mark.parametrize("captured", [False, True])
def test_training_step(captured):
    b, ids = batch(5)
    n = ids.numel()
    csr, src = tfg.tfg_build_csr(b.edge_index, n), tfg.tfg_build_csr_by_source(b.edge_index, n)
    dinv, _ = tfg.tfg_gcn_norm(csr.rowptr, csr.col, csr.perm, n, want_w_csr=False)
    gen = torch.Generator(device="cuda").manual_seed(9)
    table = torch.randn(KINDS, F, device="cuda", generator=gen)
    gamma = 1 + 0.2 * torch.randn(F, device="cuda", generator=gen)
    beta = 0.2 * torch.randn(F, device="cuda", generator=gen)
    w = torch.randn(GRAPHS, F, device="cuda", generator=gen)
    run = lambda: step(b, csr, src, dinv, ids, table, gamma, beta, w, 1.0)   # noqa: E731
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = run()
    edges = gcn_weights(b, n)
    for _ in range(3):                                         # steps of a descent: other weights each time
        if captured:
            graph.replay()
        else:
            result = run()
        pooled, grads, norm, statuses = result
        for s in statuses:
            tfg.check_status(s)
        want_pooled, want, want_norm = plain(b, edges, ids, table, gamma, beta, w, 1.0)
        assert float((pooled.double().cpu() - want_pooled).norm()) <= 2e-5 * float(want_pooled.norm())
        assert abs(float(norm) - want_norm) <= 2e-5 * want_norm
        for got, ref in zip(grads, want):
            assert float((got.double().cpu() - ref).norm()) <= 2e-5 * float(ref.norm())
        with torch.no_grad():
            for p, g in zip((table, gamma, beta), grads):
                p.sub_(0.5 * g)


def test_two_steps_at_once_on_two_streams():
    """Two batches on two streams, each with workspaces of its own, give what they give alone."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn(KINDS, F, device="cuda", generator=gen)
    gamma, beta = torch.ones(F, device="cuda"), torch.zeros(F, device="cuda")
    w = torch.randn(GRAPHS, F, device="cuda", generator=gen)
    jobs = []
    for seed in (1, 2):
        b, ids = batch(seed)
        n = ids.numel()
        csr, src = tfg.tfg_build_csr(b.edge_index, n), tfg.tfg_build_csr_by_source(b.edge_index, n)
        dinv, _ = tfg.tfg_gcn_norm(csr.rowptr, csr.col, csr.perm, n, want_w_csr=False)
        jobs.append((b, csr, src, dinv, ids, table, gamma, beta, w, 0.1))
    alone = [step(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        both = []
        for s, j in zip(streams, jobs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                both.append(step(*j))
        torch.cuda.synchronize()
        for x, y in zip(alone, both):
            assert torch.equal(x[0], y[0]) and torch.equal(x[2], y[2])
            assert all(torch.equal(p, q) for p, q in zip(x[1], y[1]))


def test_aggregation_reads_looked_up_rows():
    """bf16 rows of a table straight into the aggregation."""
    b, ids = batch(8)
    n = ids.numel()
    csr = tfg.tfg_build_csr(b.edge_index, n)
    table = torch.randn(KINDS, F, device="cuda")
    x, _ = tfg.tfg_embedding_lookup(table, ids, 0.5, padding_id=-1, out_dtype=torch.bfloat16)
    out = tfg.tfg_aggregate_sum(csr.rowptr, csr.col, x)
    ei, xs = b.edge_index.cpu(), x.double().cpu()
    ref, scale = (torch.zeros(n, F, dtype=torch.float64).index_add(0, ei[1], v[ei[0]]) for v in (xs, xs.abs()))
    assert bool(((out.double().cpu() - ref).abs() <= 1e-5 * scale).all())
