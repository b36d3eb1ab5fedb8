"""What a model puts around the aggregations, as measurable cases.

Three operators frame a training step on graphs, and each is measured as a user's program
calls it:

  embed  ids -> scaled feature rows, and the gradient of the table by sorted ids.  The ids
         are new in every pass (a new batch), so grouping them is part of a training pass.
  norm   group norm with an activation over the graphs of a batch, channels last: forward,
         or forward and backward.
  clip   the norm over all gradients of a model and the clipped gradients.

`own` False computes the plain form in elementary torch operations; True calls the
framework.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda" if torch.cuda.is_available() else "cpu"
_DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2, "int64": 8, "int32": 4}
EPS = 1e-5


def listed():
    return [
        # serving: the feature rows of a handful of queried nodes, latency bound
        {"name": "embed_serve_64_of_19717_f256", "op": "embed", "n": 64, "rows": 19717, "f": 256, "table": "fp32",
         "out": "fp32", "ids": "int64", "dist": "uniform", "pad": 0.0, "train": False},
        # training input of 1,024 molecules: 112,640 atoms of 119 kinds, a few of them most of the atoms
        {"name": "embed_atoms_112640_of_119_f128", "op": "embed", "n": 112640, "rows": 119, "f": 128, "table": "fp32",
         "out": "fp32", "ids": "int64", "dist": "zipf", "pad": 0.0, "train": True},
        # a sampled subgraph trains some rows of a table with one row per node (width without 16-byte bf16 rows)
        {"name": "embed_sampled_60000_of_169343_f100", "op": "embed", "n": 60000, "rows": 169343, "f": 100,
         "table": "fp32", "out": "bf16", "ids": "int32", "dist": "uniform", "pad": 0.0, "train": True},
        # text on nodes: padded token ids of a natural vocabulary, wide rows, bf16 storage
        {"name": "embed_tokens_131072_of_50000_f1024", "op": "embed", "n": 131072, "rows": 50000, "f": 1024,
         "table": "bf16", "out": "bf16", "ids": "int64", "dist": "zipf", "pad": 0.1, "train": True},
        # a hidden layer's norm on a small citation graph: one graph, latency bound
        {"name": "norm_citation_2708_f64", "op": "norm", "n": 2708, "graphs": 1, "sizes": "even", "f": 64, "groups": 8,
         "act": "gelu", "x": "fp32", "out": "fp32", "train": False},
        # single rows, each a graph of its own: the form for one node or token at a time
        {"name": "norm_rows_4096_f1024", "op": "norm", "n": 4096, "graphs": 4096, "sizes": "even", "f": 1024,
         "groups": 32, "act": "silu", "x": "bf16", "out": "bf16", "train": False},
        # ragged batch, odd channel counts: 300 graphs of 19,717 nodes, groups of 3 channels
        {"name": "norm_ragged_19717_f123", "op": "norm", "n": 19717, "graphs": 300, "sizes": "skew", "f": 123,
         "groups": 41, "act": "gelu", "x": "fp32", "out": "fp32", "train": True},
        # training on 1,024 molecules of 20 to 200 atoms
        {"name": "norm_molecules_112640_f128", "op": "norm", "n": 112640, "graphs": 1024, "sizes": "even", "f": 128,
         "groups": 32, "act": "silu", "x": "fp32", "out": "fp32", "train": True},
        # training on the 41 communities of a large dense graph
        {"name": "norm_communities_232965_f128", "op": "norm", "n": 232965, "graphs": 41, "sizes": "skew", "f": 128,
         "groups": 16, "act": "silu", "x": "bf16", "out": "bf16", "train": True},
        # gradients of a two-layer network: a few small matrices and vectors, latency bound
        {"name": "clip_small_6_of_100k", "op": "clip", "tensors": 6, "values": 100_000, "dtype": "fp32"},
        # a deep model with mixed storage: 148 tensors, matrices beside vectors
        {"name": "clip_deep_148_of_85M", "op": "clip", "tensors": 148, "values": 85_000_000, "dtype": "mixed"},
        # a large model's gradients in bf16
        {"name": "clip_large_60_of_1G", "op": "clip", "tensors": 60, "values": 1_000_000_000, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "norm", "clip"])
    if op == "embed":
        f = rng.choice([8 * _log_int(rng, 1, 128), rng.randint(3, 300)])
        rows = min(_log_int(rng, 16, 250_000), 51_000_000 // f)
        n = min(_log_int(rng, 1, 200_000), 134_000_000 // f)
        return {"op": op, "n": n, "rows": rows, "f": f, "table": rng.choice(["fp32", "bf16"]),
                "out": rng.choice(["fp32", "bf16"]), "ids": rng.choice(["int64", "int32"]),
                "dist": rng.choice(["uniform", "zipf"]), "pad": rng.choice([0.0, 0.1]), "train": rng.random() < 0.7}
    if op == "norm":
        per = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])                    # channels of a group
        groups = _log_int(rng, 1, min(128, 1024 // per))
        f = per * groups
        n = max(1, min(_log_int(rng, 300, 250_000), 29_800_000 // f))
        graphs = min(n, _log_int(rng, 1, 4096))
        train = rng.random() < 0.6
        if train:       # the gradient of a norm over two or three values is the rounding of what cancels in it
            graphs = max(1, min(graphs, n * per // 32))
        # the derivative of a ReLU jumps at 0, where the rounding of y decides: forward only
        act = rng.choice(["none", "silu", "gelu"] + ([] if train else ["relu"]))
        return {"op": op, "n": n, "graphs": graphs, "sizes": rng.choice(["even", "skew"]), "f": f, "groups": groups,
                "act": act, "x": rng.choice(["fp32", "bf16"]), "out": rng.choice(["fp32", "bf16"]), "train": train}
    dtype = rng.choice(["fp32", "bf16", "mixed"])
    most = 450_000_000 if dtype == "fp32" else 900_000_000
    return {"op": op, "tensors": _log_int(rng, 1, 300), "values": _log_int(rng, 2_000, most), "dtype": dtype}


# ---- sizes that follow from the case alone ---------------------------------
def _graph_sizes(case):
    """Nodes of each graph, their sum case["n"]: near one another ("even": 1 to 10 by weight,
    as molecules of 20 to 200 atoms), or a few graphs with most of the nodes ("skew")."""
    n, g = case["n"], case["graphs"]
    if n == g:
        return [1] * g
    rng = random.Random(1004)
    w = [rng.uniform(1.0, 10.0) if case["sizes"] == "even" else rng.lognormvariate(0.0, 1.2) for _ in range(g)]
    total = sum(w)
    sizes = [int(n * x / total) for x in w]
    sizes[max(range(g), key=lambda i: w[i])] += n - sum(sizes)
    return sizes


def _tensor_sizes(case):
    """Values of each gradient, their sum case["values"]: every other one a vector of a
    matrix's width (odd widths among them), the rest matrices of unequal sizes."""
    t, n = case["tensors"], case["values"]
    rng = random.Random(t)
    sizes, left = [0] * t, n
    for i in range(1, t, 2):
        sizes[i] = min(rng.choice([41, 64, 100, 128, 256, 1024]), max(0, left // t))
        left -= sizes[i]
    big = list(range(0, t, 2))
    w = [rng.uniform(0.5, 2.0) for _ in big]
    for i, x in zip(big, w):
        sizes[i] = int(left * x / sum(w)) // 8 * 8
    sizes[0] += n - sum(sizes)
    return sizes


def _tensor_dtypes(case):
    """"mixed": matrices in bf16, vectors in fp32."""
    return [case["dtype"] if case["dtype"] != "mixed" else ("bf16", "fp32")[i % 2] for i in range(case["tensors"])]


def _probabilities(case):
    v = torch.arange(case["rows"], dtype=torch.float64)
    p = 1.0 / (v + 2.7) if case["dist"] == "zipf" else torch.ones_like(v)
    return p / p.sum()


# ---- inputs ----------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _inputs(case, seed):
    g = _generator(seed)

    def normal(*shape, dtype="fp32"):
        return torch.randn(*shape, generator=g, device=DEV, dtype=_DT[dtype])

    if case["op"] == "embed":
        n, f = case["n"], case["f"]
        s = {"table": normal(case["rows"], f, dtype=case["table"])}
        u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
        cum = _probabilities(case).to(DEV).cumsum(0)
        ids = torch.searchsorted(cum, u).clamp_(max=case["rows"] - 1)
        name = torch.randperm(case["rows"], generator=g, device=DEV)        # frequent ids lie anywhere in the table
        ids = name[ids]
        s["padding"] = -1
        if case["pad"] > 0:
            ids[torch.rand(n, generator=g, device=DEV) < case["pad"]] = -1
        s["ids"] = ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)
        s["scale"] = math.sqrt(f)
        if case["train"]:
            s["grad"] = normal(n, f, dtype=case["out"])
        return s
    if case["op"] == "norm":
        n, f = case["n"], case["f"]
        sizes = torch.tensor(_graph_sizes(case), device=DEV)
        sizes = sizes[torch.randperm(case["graphs"], generator=g, device=DEV)]
        offsets = torch.zeros(case["graphs"] + 1, dtype=torch.int64, device=DEV)
        torch.cumsum(sizes, 0, out=offsets[1:])
        spread = 0.5 + torch.rand(f, generator=g, device=DEV)
        s = {"x": (normal(n, f) * spread + normal(f)).to(_DT[case["x"]]), "offsets": offsets,
             "gamma": 1.0 + 0.1 * normal(f), "beta": 0.1 * normal(f)}
        if case["train"]:
            s["grad"] = normal(n, f, dtype=case["out"])
        return s
    s = {"grads": [0.05 * normal(k, dtype=d) for k, d in zip(_tensor_sizes(case), _tensor_dtypes(case))],
         "clip": 1.0}
    # the clipped gradients go to the buffers that the optimiser reads, one per type
    start = {"fp32": [], "bf16": []}
    end = {"fp32": 0, "bf16": 0}
    for k, d in zip(_tensor_sizes(case), _tensor_dtypes(case)):
        start[d].append(end[d])
        end[d] += (k + 63) // 64 * 64
    s["flat"] = {d: torch.zeros(m, dtype=_DT[d], device=DEV) for d, m in end.items() if m}
    at = {d: iter(v) for d, v in start.items()}
    s["outs"] = [s["flat"][d].narrow(0, next(at[d]), k) if k else torch.empty(0, dtype=_DT[d], device=DEV)
                 for k, d in zip(_tensor_sizes(case), _tensor_dtypes(case))]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    return s


# ---- one pass --------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s, s["case"])


def _own(s, case):
    from paper_2101_11552_gb300 import tfg
    if case["op"] == "embed":
        out, _ = tfg.tfg_embedding_lookup(s["table"], s["ids"], s["scale"], padding_id=s["padding"],
                                          out_dtype=_DT[case["out"]])
        if not case["train"]:
            return out
        groups = tfg.tfg_group_ids(s["ids"], case["rows"], padding_id=s["padding"])
        return out, tfg.tfg_embedding_backward(groups, s["grad"], s["scale"])
    if case["op"] == "norm":
        r = tfg.tfg_group_norm(s["x"], s["offsets"], case["groups"], s["gamma"], s["beta"], eps=EPS,
                               activation=case["act"], out_dtype=_DT[case["out"]], want_stats=case["train"])
        if not case["train"]:
            return r.out
        return (r.out,) + tfg.tfg_group_norm_backward(s["x"], s["offsets"], case["groups"], s["gamma"], s["beta"],
                                                      r.mean, r.rstd, s["grad"], activation=case["act"])
    _, norm = tfg.tfg_clip_by_global_norm(s["grads"], s["clip"], outs=s["outs"])
    return {"norm": norm, **s["flat"]}


def _plain(s, case):
    if case["op"] == "embed":
        return _plain_embed(s, case)
    if case["op"] == "norm":
        return _plain_norm(s, case)
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = s["clip"] / torch.clamp(norm, min=s["clip"])
    for o, t in zip(s["outs"], s["grads"]):
        o.copy_(t.float() * factor)
    return {"norm": norm.reshape(1), **s["flat"]}


def _plain_embed(s, case):
    ids = s["ids"].long()
    here = ids != s["padding"]
    at = torch.where(here, ids, torch.zeros_like(ids))
    out = (s["table"][at].float() * s["scale"] * here[:, None]).to(_DT[case["out"]])
    if not case["train"]:
        return out
    # a frequent id's gradient is a long sum, in 64 bits
    grad = s["grad"].double() * here[:, None]
    total = torch.zeros(case["rows"], case["f"], dtype=torch.float64, device=DEV).index_add_(0, at, grad)
    return out, (total * s["scale"]).float()


def _act(y, name):
    if name == "relu":
        return torch.clamp(y, min=0.0)
    if name == "silu":
        return y / (1.0 + torch.exp(-y))
    if name == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y


def _act_slope(y, name):
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-y))
        return p * (1.0 + y * (1.0 - p))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(y * math.sqrt(0.5))) + y * torch.exp(-0.5 * y * y) / math.sqrt(2.0 * math.pi)
    if name == "relu":
        return (y > 0).float()
    return torch.ones_like(y)


def _plain_norm(s, case):
    n, f, k = case["n"], case["f"], case["groups"]
    offsets = s["offsets"]
    graph = torch.searchsorted(offsets, torch.arange(n, device=DEV), right=True) - 1
    count = torch.clamp(offsets[1:] - offsets[:-1], min=1)[:, None].float() * (f // k)

    def per_graph(v):
        """Sums over the nodes of each graph of v [n, k]: a running sum in 64 bits and its differences."""
        run_sum = torch.zeros(k, n + 1, dtype=torch.float64, device=DEV)
        torch.cumsum(v.t().double().contiguous(), 1, out=run_sum[:, 1:])
        return (run_sum[:, offsets[1:]] - run_sum[:, offsets[:-1]]).t().float()

    x = s["x"].float().reshape(n, k, f // k)
    mean = per_graph(x.sum(2)) / count
    x = x - mean[graph][:, :, None]
    rstd = 1.0 / torch.sqrt(per_graph((x * x).sum(2)) / count + EPS)
    h = x * rstd[graph][:, :, None]
    gamma, beta = s["gamma"].reshape(k, -1), s["beta"].reshape(k, -1)
    y = h * gamma + beta
    out = _act(y, case["act"]).reshape(n, f).to(_DT[case["out"]])
    if not case["train"]:
        return out
    dy = s["grad"].float().reshape(n, k, f // k) * _act_slope(y, case["act"])
    grad_beta, grad_gamma = dy.sum(0).reshape(f), (dy * h).sum(0).reshape(f)
    dh = dy * gamma
    s1, s2 = per_graph(dh.sum(2)) / count, per_graph((dh * h).sum(2)) / count
    gx = rstd[graph][:, :, None] * (dh - s1[graph][:, :, None] - h * s2[graph][:, :, None])
    return out, gx.reshape(n, f).to(_DT[case["out"]]), grad_gamma, grad_beta


# ---- the work of a pass ----------------------------------------------------
def work(case):
    if case["op"] == "embed":
        n, f, v = case["n"], case["f"], case["rows"]
        named = float((1.0 - torch.exp(-n * (1.0 - case["pad"]) * _probabilities(case))).sum())   # rows some id names
        rows = n * f * _SIZE[case["out"]]
        b = n * _SIZE[case["ids"]] + named * f * _SIZE[case["table"]] + rows
        if case["train"]:
            b += rows * (1.0 - case["pad"]) + 4 * v * f
        return {"bytes": b, "flops": (2.0 if case["train"] else 1.0) * n * f}
    if case["op"] == "norm":
        n, f, g, k = case["n"], case["f"], case["graphs"], case["groups"]
        b = n * f * (_SIZE[case["x"]] + _SIZE[case["out"]]) + 8 * (g + 1) + 8 * f
        if case["train"]:
            b += 2 * n * f * _SIZE[case["out"]] + 8 * g * k + 8 * f
        return {"bytes": b, "flops": (30.0 if case["train"] else 10.0) * n * f}
    b = sum(2 * k * _SIZE[d] for k, d in zip(_tensor_sizes(case), _tensor_dtypes(case)))
    return {"bytes": b + 4, "flops": 3.0 * case["values"]}


# ---- the definitions in 64 bits --------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "embed":
        return _exact_embed(s, case)
    if case["op"] == "norm":
        return _exact_norm(s, case)
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in s["grads"]))
    factor = s["clip"] / max(norm, s["clip"])
    flat = {d: torch.zeros(t.numel(), dtype=torch.float64, device=DEV) for d, t in s["flat"].items()}
    at = {d: 0 for d in flat}
    for t, d in zip(s["grads"], _tensor_dtypes(case)):
        if t.numel():
            flat[d][at[d]:at[d] + t.numel()] = t.double() * factor
        at[d] += (t.numel() + 63) // 64 * 64
    return {"norm": torch.tensor([norm], dtype=torch.float64), **flat}


def _exact_embed(s, case):
    ids, f = s["ids"].long(), case["f"]
    table = torch.cat([s["table"].double(), torch.zeros(1, f, dtype=torch.float64, device=DEV)])
    ids = torch.where(ids == s["padding"], case["rows"], ids)              # the row of zeros behind the table
    out = table.index_select(0, ids) * s["scale"]
    if not case["train"]:
        return out
    # each row's sum as a difference of running sums over the positions sorted by id
    order = torch.argsort(ids, stable=True)
    ends = torch.cumsum(torch.bincount(ids, minlength=case["rows"] + 1), 0)[:case["rows"]]
    run_sum = torch.zeros(case["n"] + 1, f, dtype=torch.float64, device=DEV)
    torch.cumsum(s["grad"].index_select(0, order).double(), 0, out=run_sum[1:])
    total = run_sum[ends]
    total[1:] -= run_sum[ends[:-1]]
    return out, total * s["scale"]


def _exact_norm(s, case):
    n, f, k = case["n"], case["f"], case["groups"]
    out = torch.empty(n, f, dtype=torch.float64, device=DEV)
    gx, gg, gb = torch.empty_like(out), out.new_zeros(f), out.new_zeros(f)
    gamma, beta = s["gamma"].double().reshape(k, -1), s["beta"].double().reshape(k, -1)
    ends = s["offsets"].tolist()
    for a, b in zip(ends[:-1], ends[1:]):                                   # graph by graph, as defined
        if a == b:
            continue
        x = s["x"][a:b].double().reshape(b - a, k, -1)
        mean = x.mean((0, 2), keepdim=True)
        rstd = (((x - mean) ** 2).mean((0, 2), keepdim=True) + EPS) ** -0.5
        h = (x - mean) * rstd
        y = h * gamma + beta
        if case["act"] == "relu":
            z, slope = y * (y > 0), (y > 0).double()
        elif case["act"] == "silu":
            p = torch.sigmoid(y)
            z, slope = y * p, p + y * p * (1 - p)
        elif case["act"] == "gelu":
            p = torch.special.ndtr(y)
            z, slope = y * p, p + y * torch.exp(-y * y / 2) / math.sqrt(2 * math.pi)
        else:
            z, slope = y, torch.ones_like(y)
        out[a:b] = z.reshape(b - a, f)
        if case["train"]:
            dy = s["grad"][a:b].double().reshape(b - a, k, -1) * slope
            gb += dy.sum(0).reshape(f)
            gg += (dy * h).sum(0).reshape(f)
            d = dy * gamma
            gx[a:b] = (rstd * (d - d.mean((0, 2), keepdim=True) - h * (d * h).mean((0, 2), keepdim=True))).reshape(b - a, f)
    return (out, gx, gg, gb) if case["train"] else out
