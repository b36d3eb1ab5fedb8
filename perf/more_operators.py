"""A sequence layer over the nodes of a batch and the loss that trains it, as measurable cases.

Three operators, each measured as a user's program calls it:

  norm     layer norm of node rows with the addition of the residual stream in the same pass,
           and its gradients with the stream's own gradient added.
  scan     gated linear recurrence along the rows of each sequence of a batch (a node's events,
           a graph's nodes in order), one step or a whole batch, and its gradients.
  distil   the loss against a teacher's top logits with temperature, and the logits' gradient.

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
        # serving: the rows of one step of eight requests, latency bound
        {"name": "norm_serve_8_f1024", "op": "norm", "n": 8, "f": 1024, "x": "bf16", "res": "bf16", "out": "bf16",
         "train": False},
        # a hidden layer on 19,717 nodes of an odd width
        {"name": "norm_nodes_19717_f123", "op": "norm", "n": 19717, "f": 123, "x": "fp32", "res": "none", "out": "fp32",
         "train": True},
        # training on tokens of text on nodes: bf16 branches on a residual stream held in fp32
        {"name": "norm_stream_131072_f1024", "op": "norm", "n": 131072, "f": 1024, "x": "bf16", "res": "fp32",
         "out": "bf16", "train": True},
        # wide rows, everything in bf16
        {"name": "norm_wide_8192_f8192", "op": "norm", "n": 8192, "f": 8192, "x": "bf16", "res": "bf16", "out": "bf16",
         "train": True},
        # serving: one step of 64 sequences with their states, latency bound
        {"name": "scan_step_64_f1024", "op": "scan", "n": 64, "seqs": 64, "sizes": "even", "f": 1024, "kind": "sigmoid",
         "x": "bf16", "out": "bf16", "packed": True, "state": True, "train": False},
        # training on 1,024 molecules, their atoms in order
        {"name": "scan_molecules_112640_f128", "op": "scan", "n": 112640, "seqs": 1024, "sizes": "even", "f": 128,
         "kind": "sigmoid", "x": "fp32", "out": "fp32", "packed": False, "state": False, "train": True},
        # one long sequence, few channels: the length is all there is to split
        {"name": "scan_long_131072_f256", "op": "scan", "n": 131072, "seqs": 1, "sizes": "even", "f": 256, "kind": "exp",
         "x": "bf16", "out": "fp32", "packed": False, "state": True, "train": True},
        # training on 41 sequences of unequal length, gate and input the halves of one projection
        {"name": "scan_tokens_131072_f1024", "op": "scan", "n": 131072, "seqs": 41, "sizes": "skew", "f": 1024,
         "kind": "sigmoid", "x": "bf16", "out": "bf16", "packed": True, "state": True, "train": True},
        # classes of nodes on a small citation graph, latency bound
        {"name": "distil_nodes_2708_of_41", "op": "distil", "n": 2708, "classes": 41, "k": 5, "x": "fp32", "teacher": "fp32",
         "ids": "int64", "pad": 0.1, "mask": 0.0, "tau": 2.0, "mode": "grad"},
        # an odd vocabulary in fp32, forward and backward as two calls
        {"name": "distil_odd_2500_of_49999", "op": "distil", "n": 2500, "classes": 49999, "k": 50, "x": "fp32",
         "teacher": "bf16", "ids": "int32", "pad": 0.0, "mask": 0.0, "tau": 1.0, "mode": "two"},
        # training on tokens of a natural vocabulary, a tenth of them masked
        {"name": "distil_tokens_16384_of_50000", "op": "distil", "n": 16384, "classes": 50000, "k": 64, "x": "bf16",
         "teacher": "bf16", "ids": "int32", "pad": 0.0, "mask": 0.1, "tau": 2.0, "mode": "grad"},
        # the loss alone on a held-out set of a large vocabulary
        {"name": "distil_eval_4096_of_131072", "op": "distil", "n": 4096, "classes": 131072, "k": 20, "x": "bf16",
         "teacher": "fp32", "ids": "int64", "pad": 0.0, "mask": 0.0, "tau": 1.5, "mode": "loss"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "scan", "distil"])
    types = ["fp32", "bf16"]
    if op == "norm":
        f = rng.choice([8 * _log_int(rng, 2, 2048), rng.randint(17, 1000)])
        n = max(1, min(_log_int(rng, 1, 200_000), 110_000_000 // f))
        return {"op": op, "n": n, "f": f, "x": rng.choice(types), "res": rng.choice(["none"] + types),
                "out": rng.choice(types), "train": rng.random() < 0.6}
    if op == "scan":
        f = rng.choice([8 * _log_int(rng, 1, 256), rng.randint(3, 300)])
        n = max(1, min(_log_int(rng, 1, 140_000), 110_000_000 // f))
        return {"op": op, "n": n, "seqs": min(n, _log_int(rng, 1, 4096)), "sizes": rng.choice(["even", "skew"]), "f": f,
                "kind": rng.choice(["sigmoid", "exp"]), "x": rng.choice(types), "out": rng.choice(types),
                "packed": rng.random() < 0.5, "state": rng.random() < 0.5, "train": rng.random() < 0.6}
    x = rng.choice(types)
    classes = rng.choice([_log_int(rng, 3, 1000), _log_int(rng, 1000, 200_000)])
    n = max(1, min(_log_int(rng, 1, 100_000), (380_000_000 if x == "fp32" else 760_000_000) // classes))
    return {"op": op, "n": n, "classes": classes, "k": min(classes, _log_int(rng, 1, 256)), "x": x,
            "teacher": rng.choice(types), "ids": rng.choice(["int64", "int32"]), "pad": rng.choice([0.0, 0.1]),
            "mask": rng.choice([0.0, 0.2]), "tau": rng.choice([1.0, 1.5, 2.0, 4.0]),
            "mode": rng.choice(["loss", "two", "grad", "grad"])}


# ---- inputs ----------------------------------------------------------------
def _sequence_sizes(case):
    """Rows of each sequence, their sum case["n"]: near one another ("even": 1 to 10 by weight,
    as molecules of 20 to 200 atoms), or a few with most of the rows ("skew")."""
    n, s = case["n"], case["seqs"]
    if n == s:
        return [1] * s
    rng = random.Random(2005)
    w = [rng.uniform(1.0, 10.0) if case["sizes"] == "even" else rng.lognormvariate(0.0, 1.2) for _ in range(s)]
    total = sum(w)
    sizes = [int(n * x / total) for x in w]
    sizes[max(range(s), key=lambda i: w[i])] += n - sum(sizes)
    return sizes


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(*shape, dtype="fp32"):
        return torch.randn(*shape, generator=g, device=DEV, dtype=_DT[dtype])

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    if case["op"] == "norm":
        n, f = case["n"], case["f"]
        res = None if case["res"] == "none" else normal(n, f, dtype=case["res"]).mul_(2.0)
        x = normal(n, f).mul_(0.5 + uniform(f)).add_(0.5 * normal(f)).to(_DT[case["x"]])
        s = {"x": x, "res": res, "gamma": 1.0 + 0.1 * normal(f), "beta": 0.1 * normal(f)}
        if case["train"]:
            s["grad"] = normal(n, f, dtype=case["out"])
            s["skip"] = None if res is None else normal(n, f, dtype=case["res"])
        return s
    if case["op"] == "scan":
        n, f, q = case["n"], case["f"], case["seqs"]
        sizes = torch.tensor(_sequence_sizes(case), device=DEV)
        sizes = sizes[torch.randperm(q, generator=g, device=DEV)]
        offsets = torch.zeros(q + 1, dtype=torch.int64, device=DEV)
        torch.cumsum(sizes, 0, out=offsets[1:])
        gate = normal(n, f).add_(2.5 + 1.5 * normal(f))          # memories of a few steps to a few hundred
        if case["kind"] == "exp":
            gate = gate.mul_(-1.0).exp_().mul_(-1.0)
        x = normal(n, f)
        if case["packed"]:
            both = torch.cat([gate, x], 1).to(_DT[case["x"]])
            gate, x = both[:, :f], both[:, f:]
        else:
            gate, x = gate.to(_DT[case["x"]]), x.to(_DT[case["x"]])
        s = {"gate": gate, "x": x, "offsets": offsets, "initial": normal(q, f) if case["state"] else None}
        if case["train"]:
            s["grad"] = normal(n, f, dtype=case["out"])
            s["grad_final"] = normal(q, f) if case["state"] else None
        return s
    n, v, k = case["n"], case["classes"], case["k"]
    logits = normal(n, v, dtype=case["x"]).mul_(2.0)
    part = torch.arange(k + 1, device=DEV) * v // k               # one class in each of k parts: no two alike
    width = part[1:] - part[:-1]
    ids = part[:-1] + torch.minimum((uniform(n, k) * width).long(), width - 1)
    ids = ids.gather(1, uniform(n, k).argsort(1))
    teacher = (4.0 + 2.0 * normal(n, k)).sort(1, descending=True).values
    # a student that has learnt something: its logits lean towards the teacher's
    logits.scatter_(1, ids, (0.7 * teacher + normal(n, k)).to(logits.dtype))
    if case["pad"] > 0:
        ids[uniform(n, k) < case["pad"]] = -1
    weight = torch.full((n,), 1.0 / n, device=DEV)
    weight[uniform(n) < case["mask"]] = 0.0
    s = {"logits": logits, "ids": ids.to(torch.int32 if case["ids"] == "int32" else torch.int64),
         "teacher": teacher.to(_DT[case["teacher"]]), "weight": weight}
    if case["mode"] == "two":
        s["grad_loss"] = 0.5 + uniform(n)
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
    if case["op"] == "norm":
        r = tfg.tfg_layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS, residual=s["res"], out_dtype=_DT[case["out"]],
                               want_stats=case["train"])
        out = (r.out,) if s["res"] is None else (r.out, r.sum)
        if not case["train"]:
            return out
        return out + tfg.tfg_layer_norm_backward(r.sum, s["gamma"], r.mean, r.rstd, s["grad"], grad_sum=s["skip"])
    if case["op"] == "scan":
        r = tfg.tfg_gated_recurrence(s["gate"], s["x"], s["offsets"], case["kind"], initial=s["initial"],
                                     out_dtype=_DT[case["out"]], want_final=case["state"], want_checkpoints=case["train"])
        out = (r.out, r.final) if case["state"] else (r.out,)
        if not case["train"]:
            return out
        b = tfg.tfg_gated_recurrence_backward(s["gate"], s["x"], s["offsets"], r.checkpoints, s["grad"], case["kind"],
                                              initial=s["initial"], grad_final=s["grad_final"])
        return out + (tuple(b) if case["state"] else tuple(b[:2]))
    a = (s["logits"], s["ids"], s["teacher"], case["tau"])
    if case["mode"] == "loss":
        return tfg.tfg_distillation_loss(*a, row_weight=s["weight"], padding_id=-1).loss
    if case["mode"] == "grad":
        r = tfg.tfg_distillation_loss(*a, row_weight=s["weight"], padding_id=-1, want_grad=True)
        return r.loss, r.grad_logits
    r = tfg.tfg_distillation_loss(*a, row_weight=s["weight"], padding_id=-1, want_stats=True)
    return r.loss, tfg.tfg_distillation_loss_backward(*a, r.stats, s["grad_loss"], row_weight=s["weight"], padding_id=-1)


def _plain(s, case):
    return {"norm": _plain_norm, "scan": _plain_scan, "distil": _plain_distil}[case["op"]](s, case)


def _plain_norm(s, case):
    x = s["x"].float()
    if s["res"] is not None:                      # the stream in its own type is what is normalised
        total = (x + s["res"].float()).to(s["res"].dtype)
        x = total.float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    h = c * rstd
    out = (h * s["gamma"] + s["beta"]).to(_DT[case["out"]])
    out = (out,) if s["res"] is None else (out, total)
    if not case["train"]:
        return out
    g = s["grad"].float()
    d = g * s["gamma"]
    gx = rstd * (d - d.mean(1, keepdim=True) - h * (d * h).mean(1, keepdim=True))
    kind = s["grad"].dtype
    if s["skip"] is not None:
        gx, kind = gx + s["skip"].float(), s["skip"].dtype
    # the weights' gradients are sums over all rows, in 64 bits
    return out + (gx.to(kind), (g * h).sum(0, dtype=torch.float64).float(), g.sum(0, dtype=torch.float64).float())


def _scan_in_steps(a, b):
    """v[t] = a[t] v[t - 1] + b[t] along dimension 0 for all t at once, by doubling: after the
    step for 2^j every row holds what its last 2^(j+1) rows make of the state before them."""
    step = 1
    while step < a.shape[0]:
        b[step:] = b[step:] + a[step:] * b[:-step]
        a[step:] = a[step:] * a[:-step]
        if step * 2 < a.shape[0]:
            a[:step] = 0.0                        # nothing comes before these rows
        step *= 2
    return b


def _plain_scan(s, case):
    offsets, seqs = s["offsets"], case["seqs"]
    kind, dt = case["kind"], s["x"].dtype
    has = offsets[1:] > offsets[:-1]
    first, last = offsets[:-1][has], offsets[1:][has] - 1
    # products of many decays and sums of many steps: in 64 bits
    z, x = s["gate"].double(), s["x"].double()
    if kind == "sigmoid":
        a = 1.0 / (1.0 + torch.exp(-z))
        fresh = 1.0 / (1.0 + torch.exp(z))
    else:
        a, fresh = torch.exp(z), torch.ones((), dtype=torch.float64, device=DEV)
    b = fresh * x
    state = torch.zeros(seqs, case["f"], dtype=torch.float64, device=DEV)
    if s["initial"] is not None:
        state = s["initial"].double()
    b[first] += a[first] * state[has]
    keep = a.clone()
    keep[first] = 0.0
    h = _scan_in_steps(keep, b)
    out = (h.to(_DT[case["out"]]),)
    if case["state"]:
        final = state.clone()
        final[has] = h[last]
        out += (final.float(),)
    if not case["train"]:
        return out
    back = s["grad"].double()
    if s["grad_final"] is not None:
        back[last] += s["grad_final"][has].double()
    keep = torch.zeros_like(a)
    keep[:-1] = a[1:]
    keep[last] = 0.0
    lam = _scan_in_steps(keep.flip(0), back.flip(0)).flip(0)
    before = torch.empty_like(h)
    before[1:] = h[:-1]
    before[first] = state[has]
    if kind == "sigmoid":
        gz, gx = lam * (before - x) * a * fresh, lam * fresh
    else:
        gz, gx = lam * before * a, lam
    out += (gz.to(dt), gx.to(dt))
    if case["state"]:
        g0 = s["grad_final"].double()
        g0[has] = a[first] * lam[first]
        out += (g0.float(),)
    return out


def _plain_distil(s, case):
    ids, tau = s["ids"].long(), case["tau"]
    here = (ids >= 0) & (s["weight"] != 0)[:, None]
    at = torch.where(here, ids, torch.zeros_like(ids))
    t = torch.where(here, s["teacher"].float() / tau, torch.full_like(ids, -math.inf, dtype=torch.float32))
    some = here.any(1, keepdim=True)
    top = torch.where(some, t.max(1, keepdim=True).values, torch.zeros((), device=DEV))
    e = torch.exp(t - top)
    total = torch.where(some, e.sum(1, keepdim=True), torch.ones((), device=DEV))
    p = e / total
    log_p = torch.where(here, t - top, torch.zeros((), device=DEV)) - torch.log(total)
    y = s["logits"].float() / tau
    y -= y.max(1, keepdim=True).values
    chosen = y.gather(1, at)
    y.exp_()
    norm = y.sum(1, keepdim=True)
    log_q = chosen - torch.log(norm)
    factor = s["weight"] * some[:, 0].float()
    loss = factor * tau * tau * (p * (log_p - log_q)).sum(1)
    if case["mode"] == "loss":
        return loss
    y /= norm
    y.scatter_add_(1, at, -p)
    if case["mode"] == "two":
        factor = factor * s["grad_loss"]
    y *= (factor * tau)[:, None]
    return loss, y.to(s["logits"].dtype)


# ---- the work of a pass ----------------------------------------------------
def work(case):
    if case["op"] == "norm":
        n, f = case["n"], case["f"]
        x, out = _SIZE[case["x"]], _SIZE[case["out"]]
        res = 0 if case["res"] == "none" else _SIZE[case["res"]]
        b = n * f * (x + 2 * res + out) + 8 * f
        if case["train"]:
            b += n * f * (out + (2 * res or out)) + 8 * n + 8 * f
        return {"bytes": b, "flops": (20.0 if case["train"] else 8.0) * n * f}
    if case["op"] == "scan":
        n, f = case["n"], case["f"]
        x, out, state = _SIZE[case["x"]], _SIZE[case["out"]], 4 * case["seqs"] * f if case["state"] else 0
        b = n * f * (2 * x + out) + 2 * state + 8 * (case["seqs"] + 1)
        if case["train"]:
            b += n * f * (out + 2 * x) + 2 * state
        return {"bytes": b, "flops": (20.0 if case["train"] else 8.0) * n * f}
    n, v, k = case["n"], case["classes"], case["k"]
    row = v * _SIZE[case["x"]]
    b = n * (1.0 - case["mask"]) * (row + k * (_SIZE[case["ids"]] + _SIZE[case["teacher"]])) + 8 * n
    if case["mode"] != "loss":
        b += n * row
    return {"bytes": b, "flops": (4.0 if case["mode"] == "loss" else 8.0) * n * v}


# ---- the definitions in 64 bits --------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "scan": _exact_scan, "distil": _exact_distil}[case["op"]](s, case)


def _exact_norm(s, case):
    x = s["x"].double()
    if s["res"] is not None:
        total = (x + s["res"].double()).to(s["res"].dtype).double()
        x = total
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    inverse = (var + EPS) ** -0.5
    h = (x - mean) * inverse
    out = torch.addcmul(s["beta"].double(), h, s["gamma"].double())
    out = (out,) if s["res"] is None else (out, total)
    if not case["train"]:
        return out
    g = s["grad"].double()
    d = g * s["gamma"].double()
    # the rest of d after its projections on the constant row and on h
    rest = d - d.mean(1, keepdim=True)
    rest -= h * torch.einsum("nf,nf->n", rest, h)[:, None] / case["f"]
    gx = rest * inverse
    if s["skip"] is not None:
        gx += s["skip"].double()
    return out + (gx, torch.einsum("nf,nf->f", g, h), torch.einsum("nf->f", g))


def _exact_steps(a, b):
    """v[t] = a[t] v[t - 1] + b[t] step by step, all blocks of about sqrt(T) rows side by side,
    then from block to block."""
    n, f = a.shape
    size = max(1, math.isqrt(n))
    blocks = -(-n // size)
    fill = blocks * size - n
    a = torch.cat([a, a.new_ones(fill, f)]).reshape(blocks, size, f)
    b = torch.cat([b, b.new_zeros(fill, f)]).reshape(blocks, size, f)
    v, product = torch.empty_like(b), torch.empty_like(a)
    v[:, 0], product[:, 0] = b[:, 0], a[:, 0]
    for t in range(1, size):
        v[:, t] = a[:, t] * v[:, t - 1] + b[:, t]
        product[:, t] = a[:, t] * product[:, t - 1]
    for i in range(1, blocks):
        v[i] += product[i] * v[i - 1, -1]
    return v.reshape(-1, f)[:n]


def _exact_scan(s, case):
    ends = s["offsets"].tolist()
    z, x = s["gate"].double(), s["x"].double()
    if case["kind"] == "sigmoid":
        a, fresh = torch.sigmoid(z), torch.sigmoid(-z)
    else:
        a, fresh = z.exp(), torch.ones_like(z)
    state = torch.zeros(case["seqs"], case["f"], dtype=torch.float64, device=DEV)
    if s["initial"] is not None:
        state = s["initial"].double()
    rows = [(i, p, q) for i, (p, q) in enumerate(zip(ends[:-1], ends[1:])) if q > p]
    at = torch.tensor([i for i, _, _ in rows], device=DEV)
    starts = torch.tensor([p for _, p, _ in rows], device=DEV)
    stops = torch.tensor([q - 1 for _, _, q in rows], device=DEV)
    # a sequence's first step forgets all rows before it and begins with its state
    chain, add = a.clone(), fresh * x
    add.index_add_(0, starts, a[starts] * state[at])
    chain[starts] = 0.0
    h = _exact_steps(chain, add)
    out = (h,)
    if case["state"]:
        out += (state.index_copy(0, at, h[stops]),)
    if not case["train"]:
        return out
    # backwards: the adjoint of row t takes a[t + 1] of the next row's, within the sequence
    grad = s["grad"].double()
    if s["grad_final"] is not None:
        grad = grad.index_add(0, stops, s["grad_final"].double()[at])
    chain = torch.cat([a[1:], torch.zeros_like(a[:1])])
    chain[stops] = 0.0
    adjoint = _exact_steps(chain.flip(0), grad.flip(0)).flip(0)
    h_before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    h_before[starts] = state[at]
    # dh/dz = h_before da/dz + x dfresh/dz
    if case["kind"] == "sigmoid":
        slope = a * fresh
        gz = adjoint * (h_before * slope - x * slope)
    else:
        gz = adjoint * h_before * a
    out += (gz, adjoint * fresh)
    if case["state"]:
        out += (s["grad_final"].double().index_copy(0, at, adjoint[starts] * a[starts]),)
    return out


def _exact_distil(s, case):
    n, v, tau = case["n"], case["classes"], case["tau"]
    loss = torch.zeros(n, dtype=torch.float64, device=DEV)
    grad = None if case["mode"] == "loss" else torch.zeros(n, v, dtype=torch.float64, device=DEV)
    for a in range(0, n, 1024):
        r = slice(a, min(n, a + 1024))
        ids, w = s["ids"][r].long(), s["weight"][r].double()
        log_p = torch.log_softmax((s["teacher"][r].double() / tau).masked_fill(ids < 0, -math.inf), 1)
        valid = (ids >= 0) & (w != 0)[:, None]
        log_q = torch.log_softmax(s["logits"][r].double() / tau, 1)
        p = torch.where(valid, log_p.exp(), 0.0)
        terms = torch.where(valid, p * (log_p - log_q.gather(1, ids.clamp(min=0))), 0.0)
        loss[r] = w * tau ** 2 * terms.sum(1)
        if grad is not None:
            c = w * tau * (valid.any(1))
            if case["mode"] == "two":
                c = c * s["grad_loss"][r].double()
            grad[r] = log_q.exp().scatter_add(1, ids.clamp(min=0), -p) * c[:, None]
    return loss if grad is None else (loss, grad)
