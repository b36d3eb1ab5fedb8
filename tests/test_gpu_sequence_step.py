"""Layer norm with the residual stream, gated recurrence, graph aggregation and distillation run
together as a training step of a small student on sequences does, eager and captured, against
the same step in 64 bits under autograd on the CPU; then as a serving loop, on two
streams, in two captured graphs with one workspace, and in the bounds-checked build.

The step, for nodes in order along the sequences of a batch:
  x = E[ids];  h = LN1(x);  [z | u] = h W1;  y = recurrence(z, u);  s = x + y W2;  h2 = LN2(s)
  logits = (Ahat h2) W3;  loss = sum of distillation losses of the rows
The products are torch's in fp32.  Every operator's own test bounds its error; here gradients are held
to 3e-5 of their 2-norm: a chain of ten fp32 steps, each within a few 1e-6.
"""
import gc
import os

import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import build, graphgen as gg, tfg
from _helpers import dev

pytestmark = pytest.mark.gpu
KINDS, F, CLASSES, TOP = 30, 48, 61, 7
EPS, TAU = 1e-5, 1.5


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()
    torch.backends.cuda.matmul.allow_tf32 = False
    yield
    gc.collect()                                             # exceptions that tests kept, and the tensors in their frames
    torch.cuda.empty_cache()


def batch(seed, graphs=9):
    rng = np.random.default_rng(seed)
    sizes = rng.integers(1, 150, graphs)
    sizes[graphs // 2] = 0
    n = int(sizes.sum())
    parts = [gg.with_self_loops(gg.symmetrise(gg.er_pairs(int(s), max(int(s) - 1, 0), rng)), int(s)) if s > 1
             else np.zeros((2, int(s)), np.int64) for s in sizes]
    stacked = np.ascontiguousarray(np.concatenate(parts, axis=1))
    b = tfg.tfg_batch_graphs(dev(sizes.astype(np.int64)), dev(np.array([p.shape[1] for p in parts], np.int64)), dev(stacked), n)
    tfg.check_status(b.status)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, KINDS, (n,), device="cuda", generator=gen)
    top = torch.rand(n, CLASSES, device="cuda", generator=gen).argsort(1)[:, :TOP].contiguous()
    top[torch.rand(n, TOP, device="cuda", generator=gen) < 0.1] = -1
    teacher = 2.0 * torch.randn(n, TOP, device="cuda", generator=gen)
    weight = (torch.rand(n, device="cuda", generator=gen) > 0.2).float() / n
    return b, n, ids, top, teacher, weight


def weights(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def normal(*shape, scale):
        return scale * torch.randn(*shape, device="cuda", generator=gen)
    return {"table": normal(KINDS, F, scale=1.0), "g1": 1 + normal(F, scale=0.2), "b1": normal(F, scale=0.2),
            "w1": normal(F, 2 * F, scale=F ** -0.5), "w2": normal(F, F, scale=F ** -0.5), "g2": 1 + normal(F, scale=0.2),
            "b2": normal(F, scale=0.2), "w3": normal(F, CLASSES, scale=F ** -0.5)}


class Job:
    def __init__(self, seed):
        self.b, self.n, self.ids, self.top, self.teacher, self.weight = batch(seed)
        self.w = weights(seed + 100)
        self.csr, self.src = tfg.tfg_build_csr(self.b.edge_index, self.n), tfg.tfg_build_csr_by_source(self.b.edge_index, self.n)
        self.dinv, _ = tfg.tfg_gcn_norm(self.csr.rowptr, self.csr.col, self.csr.perm, self.n, want_w_csr=False)
        self.groups = tfg.tfg_group_ids(self.ids, KINDS)

    def step(self):
        w, off = self.w, self.b.node_offsets
        x, _ = tfg.tfg_embedding_lookup(w["table"], self.ids)
        l1 = tfg.tfg_layer_norm(x, w["g1"], w["b1"], EPS)
        zu = l1.out @ w["w1"]
        z, u = zu[:, :F], zu[:, F:]
        r = tfg.tfg_gated_recurrence(z, u, off)
        l2 = tfg.tfg_layer_norm(r.out @ w["w2"], w["g2"], w["b2"], EPS, residual=x)
        a = tfg.tfg_gcn_aggregate_sum(self.csr.rowptr, self.csr.col, self.dinv, l2.out)
        logits = a @ w["w3"]
        d = tfg.tfg_distillation_loss(logits, self.top, self.teacher, TAU, row_weight=self.weight, padding_id=-1, want_grad=True)
        g = {"w3": a.t() @ d.grad_logits}
        ga = tfg.tfg_gcn_aggregate_backward(self.src, self.dinv, d.grad_logits @ w["w3"].t())
        gs, g["g2"], g["b2"] = tfg.tfg_layer_norm_backward(l2.sum, w["g2"], l2.mean, l2.rstd, ga)
        g["w2"] = r.out.t() @ gs
        gzu = torch.empty_like(zu)
        status = torch.empty(1, dtype=torch.int32, device="cuda")
        tfg.tfg_gated_recurrence_backward(z, u, off, r.checkpoints, gs @ w["w2"].t(), grad_gate=gzu[:, :F], grad_x=gzu[:, F:],
                                          status=status)
        g["w1"] = l1.out.t() @ gzu
        gx, g["g1"], g["b1"] = tfg.tfg_layer_norm_backward(x, w["g1"], l1.mean, l1.rstd, gzu @ w["w1"].t(), grad_sum=gs)
        g["table"] = tfg.tfg_embedding_backward(self.groups, gx)
        names = sorted(g)
        clipped, norm = tfg.tfg_clip_by_global_norm([g[k].contiguous() for k in names], 1e6)
        return d.loss, dict(zip(names, clipped)), norm, [r.status, status, d.status]

    def plain(self):
        w = {k: v.double().cpu().requires_grad_() for k, v in self.w.items()}
        ids, off, top = self.ids.cpu(), self.b.node_offsets.tolist(), self.top.cpu()
        def norm(s, g, b):
            c = s - s.mean(1, keepdim=True)
            return c / torch.sqrt((c ** 2).mean(1, keepdim=True) + EPS) * g + b
        x = w["table"][ids]
        zu = norm(x, w["g1"], w["b1"]) @ w["w1"]
        a, u = torch.sigmoid(zu[:, :F]), zu[:, F:]
        rows = []
        for p, q in zip(off, off[1:]):
            v = torch.zeros(F, dtype=torch.float64)
            for t in range(p, q):
                v = a[t] * v + (1 - a[t]) * u[t]
                rows.append(v)
        h2 = norm(x + torch.stack(rows) @ w["w2"], w["g2"], w["b2"])
        ei = self.b.edge_index.cpu()
        deg = torch.zeros(self.n, dtype=torch.float64).index_add(0, ei[1], torch.ones(ei.shape[1], dtype=torch.float64))
        weight = (deg[ei[0]] * deg[ei[1]]) ** -0.5
        agg = torch.zeros(self.n, F, dtype=torch.float64).index_add(0, ei[1], h2[ei[0]] * weight[:, None])
        log_q = torch.log_softmax(agg @ w["w3"] / TAU, 1)
        here = top >= 0
        log_p = torch.log_softmax((self.teacher.double().cpu() / TAU).masked_fill(~here, -float("inf")), 1)
        terms = torch.where(here, log_p.exp() * (torch.where(here, log_p, 0.0) - log_q.gather(1, top.clamp(min=0))), 0.0)
        loss = self.weight.double().cpu() * TAU ** 2 * terms.sum(1)
        loss.sum().backward()
        return loss.detach(), {k: v.grad for k, v in w.items()}


def capture(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = fn()
    return graph, result


@pytest.mark.parametrize("captured", [False, True])
def test_training_step(captured):
    job = Job(3)
    if captured:
        graph, result = capture(job.step)
    for _ in range(3):                                       # steps of a descent: other weights each time
        if captured:
            graph.replay()
        else:
            result = job.step()
        loss, grads, norm, statuses = result
        for s in statuses:
            tfg.check_status(s)
        want_loss, want = job.plain()
        assert float((loss.double().cpu() - want_loss).norm()) <= 3e-5 * float(want_loss.norm())
        for k, ref in want.items():
            assert float((grads[k].double().cpu() - ref).norm()) <= 3e-5 * float(ref.norm()), k
        with torch.no_grad():
            for k, g in grads.items():
                job.w[k].sub_(0.3 * g)


def same(a, b):
    return torch.equal(a[0], b[0]) and all(torch.equal(a[1][k], b[1][k]) for k in a[1])


def test_two_steps_at_once_on_two_streams():
    jobs = [Job(1), Job(2)]
    alone = [j.step() for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        both = []
        for s, j in zip(streams, jobs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                both.append(j.step())
        torch.cuda.synchronize()
        assert all(same(x, y) for x, y in zip(alone, both))


def test_two_graphs_with_one_workspace():
    """Captured recurrences of different sizes that share a workspace, replayed in turn: what one
    leaves in it does not reach the other."""
    f = 72
    gen = torch.Generator(device="cuda").manual_seed(1)
    cases = []
    for n, cuts in ((9000, [0, 9000]), (5000, [0, 3, 4200, 5000])):
        z, x, g = (torch.randn(n, f, device="cuda", generator=gen) for _ in range(3))
        cases.append((z + 2, x, torch.tensor(cuts, device="cuda"), g))
    space = torch.full((tfg.tfg_gated_recurrence_workspace_size(9000, f),), 255, dtype=torch.uint8, device="cuda")

    def both(z, x, off, g, workspace):
        r = tfg.tfg_gated_recurrence(z, x, off, workspace=workspace)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, workspace=workspace)
        return r.out, r.final, b.gate, b.x

    want = [[t.clone() for t in both(*c, None)] for c in cases]
    made = [capture(lambda c=c: both(*c, space)) for c in cases]
    for _ in range(4):
        for (graph, got), ref in zip(made, want):
            for t in got:
                t.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_serving_loop_captured():
    """One step of 33 sequences in a captured graph, the states handed on outside of it, against the
    whole sequences at once."""
    seqs, n, f = 33, 12, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    zu = torch.randn(seqs, n, 2 * f, device="cuda", generator=gen).bfloat16()
    gamma = torch.linspace(0.5, 1.5, f, device="cuda")
    steps = torch.arange(seqs + 1, device="cuda")
    row, state, stream = zu[:, 0].clone(), torch.zeros(seqs, f, device="cuda"), torch.zeros(seqs, f, device="cuda")

    def step():
        r = tfg.tfg_gated_recurrence(row[:, :f], row[:, f:], steps, initial=state, out_dtype=torch.float32, want_checkpoints=False)
        return r, tfg.tfg_layer_norm(r.out, gamma, None, residual=stream, want_stats=False)

    graph, (r, h) = capture(step)
    outs = []
    for t in range(n):
        row.copy_(zu[:, t])
        graph.replay()
        outs.append(h.out.clone())
        state.copy_(r.final)
    flat = zu.reshape(seqs * n, 2 * f)
    whole = tfg.tfg_gated_recurrence(flat[:, :f], flat[:, f:], torch.arange(seqs + 1, device="cuda") * n, out_dtype=torch.float32)
    want = tfg.tfg_layer_norm(whole.out, gamma, None).out.view(seqs, n, f)
    # states within 12 rows' roundings of one another, divided by a spread of at least 0.05
    assert bool(((torch.stack(outs, 1) - want).abs() <= 1e-4).all())


def test_bounds_checked_build():
    path = os.path.join(build.OBJ_DIR, "libtfg_checked.so")
    newest = max(os.path.getmtime(p) for p in build._deps())
    if not os.path.exists(path) or os.path.getmtime(path) < newest:
        build.build_library(defines=("TFG_CHECK_BOUNDS=1",), lib_path=path)
    job = Job(4)
    want = job.step()
    tfg.use_library(path)
    try:
        assert same(job.step(), want)
        # inside one allocation, so that even a launch would stay within it: buffers that end
        # where the allocation does are refused when a call says that they hold more
        gc.collect()
        torch.cuda.empty_cache()
        buf = torch.zeros((32 << 20) // 4, device="cuda")
        seg = [s for s in torch.cuda.memory_snapshot()
               if s["address"] <= buf.data_ptr() < s["address"] + s["total_size"]]
        if not seg or seg[0]["address"] + seg[0]["total_size"] != buf.data_ptr() + buf.numel() * 4:
            pytest.skip("the caching allocator did not give the buffer a segment of its own")
        at, end = buf.data_ptr(), buf.data_ptr() + buf.numel() * 4
        rc = tfg.lib().tfg_layer_norm(end - 4 * 160, 0, None, 0, None, 11, 16, None, None, 1e-5, at, 0, None, None, None)
        assert rc == tfg.TFG_ERR_INDEX_RANGE and "x must hold" in tfg.tfg_last_error()
    finally:
        tfg.use_library(build.LIB_PATH)


def test_tensors_of_different_devices_are_refused():
    """Tensors of different devices are refused by name before anything runs."""
    x = torch.randn(4, 8, device="cuda")
    with pytest.raises(ValueError):
        tfg.tfg_layer_norm(x, residual=x.cpu())
    with pytest.raises(ValueError):
        tfg.tfg_gated_recurrence(x, x, torch.tensor([0, 4]))
    with pytest.raises(ValueError):
        tfg.tfg_distillation_loss(x, torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2, device="cuda"))
