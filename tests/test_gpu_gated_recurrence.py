"""Gated linear recurrence, forward and backward, against a step-by-step form in 64 bits.

Tolerances are first-order error bounds carried along the recurrence in 64 bits, u = 2^-24.  Let
M_t = a_t M_{t-1} + |b_t| be the size of what adds up to v_t.  Every row costs a few roundings of
values of at most that size, and so does every border of a thread's rows, a tile or a
window, of which there are fewer than rows: 8 u M_t in all.  1 - a = p is off by ep = (|z| + 6) u p with
the sigmoid gate (the first |z| times a, as p hangs on e^z no more than that); with the exp gate by 4 u p near 0 and (|z| + 4) u a + 2 u elsewhere.  So
  E_t = a_t E_{t-1} + 8 u M_t + ep (M_{t-1} + |x_t|)              (exp gate: no |x_t|)
and for the adjoint, of size L_t = |g_t| + a_{t+1} L_{t+1},
  F_t = (a F + ep L)_{t+1} + 8 u L_t
  grad_x:    F p + L (ep + 2 u p)                                 (exp gate: F)
  grad_gate: F (M_{t-1} + |x|) a p + L E_{t-1} a p + L (M_{t-1} + |x|) (ep + 6 u a p + u p)
  (exp gate: F M a + L E a + L M (ep + 4 u a + u))
  grad_initial: a F + L (ep + 2 u)
A result stored in bf16 adds half a step, 2^-8 of it.  Below 2^-126 the roundings above are no longer
relative: a value there is off by half a step of 2^-149 each time, 10^4 rows of four such roundings by
less than 1e-40 (met where only the final state has a gradient and 380 rows of gates lie between).
"""
import gc
import pytest
import torch

from paper_2101_11552_gb300 import tfg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
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
    tol = tol + 1e-40
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    off = (got.double().cpu() - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {(off / tol.clamp(min=1e-300)).max():.3g} of the bound, first {bad.nonzero()[:3].tolist()}"


class Plain:
    """Values and bounds of a batch, row by row on the CPU (offsets: a list)."""

    def __init__(self, z, x, offsets, kind, initial):
        z, x = z.double().cpu(), x.double().cpu()
        n, f = z.shape
        self.offsets, self.kind = offsets, kind
        seqs = len(offsets) - 1
        zero = torch.zeros(f, dtype=torch.float64)
        state = torch.zeros(seqs, f, dtype=torch.float64) if initial is None else initial.double().cpu()
        if kind == "sigmoid":
            self.a, self.p = torch.sigmoid(z), torch.sigmoid(-z)
            self.ep = (self.a * z.abs().clamp(max=200) + 6) * U * self.p + 1e-37
            b, bx = self.p * x, x.abs()
        else:
            self.a, self.p = torch.exp(z), -torch.expm1(z)
            far = (z.clamp(min=-200).abs() + 4) * U * self.a + 2 * U
            self.ep = torch.where(z.abs() <= 0.35, 4 * U * self.p.abs(), far)
            b, bx = x, torch.zeros_like(x)
        self.x, self.bx = x, bx
        self.v, self.before, self.m, self.m_before, self.e, self.e_before = (torch.zeros(n, f, dtype=torch.float64) for _ in range(6))
        self.final, self.final_tol = state.clone(), torch.zeros_like(state)
        for s, (p, q) in enumerate(zip(offsets, offsets[1:])):
            v, m, e = state[s], state[s].abs(), zero
            for t in range(p, q):
                self.before[t], self.m_before[t], self.e_before[t] = v, m, e
                e = self.a[t] * e + self.ep[t] * (m + bx[t])
                v = self.a[t] * v + b[t]
                m = self.a[t] * m + b[t].abs()
                e = e + 8 * U * m
                self.v[t], self.m[t], self.e[t] = v, m, e
            if q > p:
                self.final[s], self.final_tol[s] = v, e
        self.rows = [t for p, q in zip(offsets, offsets[1:]) for t in range(p, q)]

    def backward(self, g, g_final):
        n, f = self.a.shape
        g = torch.zeros(n, f, dtype=torch.float64) if g is None else g.double().cpu()
        last = torch.zeros_like(self.final) if g_final is None else g_final.double().cpu()
        lam, size, err = (torch.zeros(n, f, dtype=torch.float64) for _ in range(3))
        first, first_tol = last.clone(), torch.zeros_like(last)
        for s, (p, q) in enumerate(zip(self.offsets, self.offsets[1:])):
            c, l, e = last[s], last[s].abs(), torch.zeros(f, dtype=torch.float64)
            for t in range(q - 1, p - 1, -1):
                lam[t], size[t] = g[t] + c, g[t].abs() + l
                err[t] = e + 8 * U * size[t]
                c, l, e = self.a[t] * lam[t], self.a[t] * size[t], self.a[t] * err[t] + self.ep[t] * size[t]
            if q > p:
                first[s], first_tol[s] = c, e + 2 * U * size[p]
        a, p, ep, m = self.a, self.p, self.ep, self.m_before
        if self.kind == "sigmoid":
            gx, gx_tol = lam * p, err * p + size * (ep + 2 * U * p)
            way = m + self.bx
            gz = lam * (self.before - self.x) * a * p
            gz_tol = err * way * a * p + size * self.e_before * a * p + size * way * (ep + 6 * U * a * p + U * p)
        else:
            gx, gx_tol = lam, err
            gz = lam * self.before * a
            gz_tol = err * m * a + size * self.e_before * a + size * m * (ep + 4 * U * a + U)
        return (gz, gz_tol), (gx, gx_tol), (first, first_tol)


def batch(n, f, kind, dt, seed, packed=False, wide=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = 2.0 + wide * torch.randn(n, f, device="cuda", generator=gen)
    if kind == "exp":
        z = -torch.exp(-z)
    x = torch.randn(n, f, device="cuda", generator=gen)
    if packed:
        both = torch.cat([z, x], 1).to(DT[dt])
        return both[:, :f], both[:, f:]
    return z.to(DT[dt]), x.to(DT[dt])


def normal(n, f, seed, dt="f32"):
    return torch.randn(n, f, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(DT[dt])


def check(z, x, offsets, kind, initial, out_dt, g, g_final):
    n, f = z.shape
    off = torch.tensor(offsets, device="cuda")
    mark = 3.5
    out = torch.full((n, f), mark, dtype=DT[out_dt], device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off, kind, initial=initial, out=out)
    tfg.check_status(r.status)
    p = Plain(z, x, offsets, kind, initial)
    rows = p.rows
    close(r.out[rows], p.v[rows], p.e[rows], "out")
    close(r.final, p.final, p.final_tol, "final")
    idle = [t for t in range(n) if t < offsets[0] or t >= offsets[-1]]
    assert bool((r.out[idle] == mark).all()), "rows outside the sequences are left as they were"
    gz, gx = (torch.full((n, f), mark, dtype=z.dtype, device="cuda") for _ in range(2))
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, initial=initial, grad_final=g_final, want_initial=True,
                                          grad_gate=gz, grad_x=gx, status=status)
    tfg.check_status(status)
    (wz, tz), (wx, tx), (wi, ti) = p.backward(g, g_final)
    close(b.gate[rows], wz[rows], tz[rows], "grad_gate")
    close(b.x[rows], wx[rows], tx[rows], "grad_x")
    close(b.initial, wi, ti, "grad_initial")
    assert bool((gz[idle] == mark).all()) and bool((gx[idle] == mark).all())
    return r, b


KINDS = ["sigmoid", "exp"]
LAYOUTS = {                                # offsets; rows behind the last belong to no sequence
    "one row": [0, 1],
    "steps": list(range(0, 41)),
    "empty ones": [0, 0, 0, 5, 5, 9, 9, 130, 130, 131, 131],
    "padded": [7, 50, 50, 170],
    "one tile": [0, 128],
    "tile and a row": [0, 129],
    "tile borders": [0, 127, 128, 129, 256, 383, 384, 640],
    "across tiles": [0, 300, 301, 700, 1100],
    "into a window": [0, 4096],
    "past a window": [0, 4097],
    "windows": [3, 200, 8500, 8501, 12_700],
}


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f,dt", [(8, "f32"), (3, "bf16"), (72, "bf16")])
def test_layouts(layout, kind, f, dt):
    offsets = LAYOUTS[layout]
    n = offsets[-1] + (11 if layout in ("padded", "windows") else 0)
    z, x = batch(n, f, kind, dt, 1, packed=layout in ("across tiles", "windows"))
    s = len(offsets) - 1
    check(z, x, offsets, kind, normal(s, f, 2), dt, normal(n, f, 3, dt), normal(s, f, 4))


@pytest.mark.parametrize("f", [1, 2, 4, 5, 8, 16, 31, 32, 33, 64, 65, 72, 100, 136, 260])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_widths(f, dt, kind):
    offsets = [0, 1, 60, 61, 61, 290, 333]
    z, x = batch(333, f, kind, dt, f)
    check(z, x, offsets, kind, None, "f32", normal(333, f, 3, "f32"), None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("f", [40, 27])
def test_types_and_strides(dt, out, packed, f):
    offsets = [0, 200, 450]
    z, x = batch(450, f, "sigmoid", dt, 5, packed)
    check(z, x, offsets, "sigmoid", normal(2, f, 1), out, normal(450, f, 3, out), normal(2, f, 2))


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_into_one_projection(kind):
    """Inputs and gradients as halves of [N, 2F] buffers, an odd width among them."""
    for f in (32, 13):
        off = torch.tensor([0, 100, 400], device="cuda")
        z, x = batch(400, f, kind, "bf16", 2, packed=True)
        r = tfg.tfg_gated_recurrence(z, x, off, kind)
        g = normal(400, f, 3, "bf16")
        apart = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind)
        both = torch.zeros(400, 2 * f, dtype=torch.bfloat16, device="cuda")
        tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, grad_gate=both[:, :f], grad_x=both[:, f:])
        assert torch.equal(both, torch.cat([apart.gate, apart.x], 1)) and apart.initial is None


@pytest.mark.parametrize("kind", KINDS)
def test_long_memory(kind):
    """Gates near 1: 1 - a of 1e-4 to 1e-6 keeps its digits over 9,000 rows (the bound E_t grows
    with the memory only as the roundings do)."""
    n, f = 9000, 5
    z = torch.linspace(9.2, 13.8, f, device="cuda").expand(n, f).contiguous()
    if kind == "exp":
        z = -torch.exp(-z)
    x = normal(n, f, 1) + 1.0
    check(z, x, [0, n], kind, normal(1, f, 2), "f32", normal(n, f, 3), normal(1, f, 4))


@pytest.mark.parametrize("kind", KINDS)
def test_gates_at_their_ends(kind):
    n, f = 300, 16
    z, x = batch(n, f, kind, "f32", 1)
    z[40] = z[200] = -float("inf")                          # forgets
    z[90, ::2] = -80.0
    z[91] = 0.0
    if kind == "sigmoid":
        z[101] = float("inf")                                # keeps
        z[120] = 90.0
    z[60] = -0.35
    z[61] = -0.350001
    init = normal(1, f, 2) * 1e6
    r, _ = check(z, x, [0, n], kind, init, "f32", normal(n, f, 3), normal(1, f, 4))
    assert torch.equal(r.out[40], x[40]) and torch.equal(r.out[200], x[200])
    if kind == "sigmoid":
        assert torch.equal(r.out[101], r.out[100])


@pytest.mark.parametrize("lengths", [[50, 60, 70], [400, 500, 30], [5000, 300, 4200]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_no_leak_between_sequences(lengths, bad):
    """What is no number in a sequence, or its state, leaves the others as they are, bit for bit."""
    offsets = [0]
    for k in lengths:
        offsets.append(offsets[-1] + k)
    n, f = offsets[-1], 40
    off = torch.tensor(offsets, device="cuda")
    z, x = batch(n, f, "sigmoid", "f32", 1)
    init, g, gf = normal(3, f, 2), normal(n, f, 3), normal(3, f, 4)

    def run():
        r = tfg.tfg_gated_recurrence(z, x, off, "sigmoid", initial=init)
        return r, tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, "sigmoid", initial=init, grad_final=gf)

    want, want_b = run()
    want, want_b = [t.clone() for t in want[:2]], [t.clone() for t in want_b]
    mid = slice(offsets[1], offsets[2])
    x[offsets[1] + 3, 5] = bad
    g[offsets[2] - 4, 6] = bad
    init[1, 7] = bad
    gf[1, 8] = bad
    got, got_b = run()
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[mid] = False
    assert torch.equal(got.out[rest], want[0][rest]) and torch.equal(got.final[[0, 2]], want[1][[0, 2]])
    assert torch.equal(got_b.gate[rest], want_b[0][rest]) and torch.equal(got_b.x[rest], want_b[1][rest])
    assert torch.equal(got_b.initial[[0, 2]], want_b[2][[0, 2]])
    others = [c for c in range(f) if c not in (5, 6, 7, 8)]
    assert torch.equal(got.out[mid][:, others], want[0][mid][:, others])
    assert not bool(torch.isfinite(got.out[offsets[1] + 3, 5])) and not bool(torch.isfinite(got.out[offsets[1], 7]))


def test_one_step_at_a_time():
    """A sequence continued row by row, and in pieces, against the whole."""
    n, f, seqs = 70, 64, 5
    z, x = batch(n * seqs, f, "sigmoid", "bf16", 1)
    whole = [k * n for k in range(seqs + 1)]
    p = Plain(z, x, whole, "sigmoid", None)
    state = torch.zeros(seqs, f, device="cuda")
    steps = torch.arange(seqs + 1, device="cuda")
    z3, x3 = z.view(seqs, n, f), x.view(seqs, n, f)
    for t in range(n):
        r = tfg.tfg_gated_recurrence(z3[:, t], x3[:, t], steps, initial=state, out_dtype=torch.float32, want_checkpoints=False)
        at = [k * n + t for k in range(seqs)]
        close(r.out, p.v[at], p.e[at], f"step {t}")
        assert torch.equal(r.out, r.final)
        state = r.final
    state = None
    for a, b in ((0, 1), (1, 33), (33, 33), (33, 70)):
        cut = torch.arange(seqs + 1, device="cuda") * (b - a)
        r = tfg.tfg_gated_recurrence(z3[:, a:b].reshape(-1, f), x3[:, a:b].reshape(-1, f), cut, initial=state)
        state = r.final
    at = [k * n + n - 1 for k in range(seqs)]
    close(state, p.v[at], p.e[at], "pieces")


@pytest.mark.parametrize("seqs", [3000, 9000])
def test_very_many_sequences(seqs):
    gen = torch.Generator().manual_seed(seqs)
    sizes = torch.randint(0, 4, (seqs,), generator=gen)
    sizes[seqs // 2] = 500
    offsets = [0] + torch.cumsum(sizes, 0).tolist()
    n = offsets[-1]
    z, x = batch(n, 8, "exp", "f32", 1)
    check(z, x, offsets, "exp", normal(seqs, 8, 2), "f32", normal(n, 8, 3), normal(seqs, 8, 4))
    empty = [0] * (seqs + 1)
    r = tfg.tfg_gated_recurrence(z[:0], x[:0], torch.tensor(empty, device="cuda"), "exp", initial=normal(seqs, 8, 2))
    tfg.check_status(r.status)
    assert torch.equal(r.final, normal(seqs, 8, 2))


def test_final_states_alone():
    n, f = 500, 24
    z, x = batch(n, f, "sigmoid", "f32", 1)
    check(z, x, [0, 120, 500], "sigmoid", None, "f32", None, normal(2, f, 4))
    off = torch.tensor([0, 120, 500], device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints)
    assert bool((b.gate == 0).all()) and bool((b.x == 0).all())


@pytest.mark.parametrize("offsets", [[0, 50, 40, 300], [0, 100, 301], [-1, 100, 300], [5, 1 << 40, 300], [-(1 << 62), 1 << 62, 0]])
def test_bad_offsets_are_reported(offsets):
    z, x = batch(300, 33, "sigmoid", "f32", 1)
    off = torch.tensor(offsets, device="cuda")
    s = len(offsets) - 1
    r = tfg.tfg_gated_recurrence(z, x, off, initial=normal(s, 33, 1))
    assert int(r.status) == tfg.TFG_ERR_INDEX_RANGE
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, x, initial=normal(s, 33, 1), status=status)
    assert int(status) == tfg.TFG_ERR_INDEX_RANGE


def test_same_bits_every_time():
    n, f = 40_000, 200
    z, x = batch(n, f, "sigmoid", "bf16", 1)
    off = torch.tensor([0, 17, 30_000, n], device="cuda")
    g = normal(n, f, 2, "bf16")
    runs = []
    for _ in range(6):
        r = tfg.tfg_gated_recurrence(z, x, off)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g)
        runs.append((r.out, r.final, r.checkpoints, b.gate, b.x))
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


@pytest.mark.parametrize("kind", KINDS)
def test_gradient_is_the_slope(kind):
    """<grad, u> against central differences of the 64-bit form (step 1e-4: an error of 1e-8)."""
    n, f, offsets = 30, 4, [0, 11, 30]
    z, x = (t.double() for t in batch(n, f, kind, "f32", 1, wide=0.5))
    init, g, gf = normal(2, f, 2).double(), normal(n, f, 3), normal(2, f, 4)
    off = torch.tensor(offsets, device="cuda")

    def loss(z, x, init):
        total = 0.0
        a = torch.sigmoid(z) if kind == "sigmoid" else torch.exp(z)
        for s, (p, q) in enumerate(zip(offsets, offsets[1:])):
            v = init[s]
            for t in range(p, q):
                v = a[t] * v + ((1 - a[t]) * x[t] if kind == "sigmoid" else x[t])
                total += float((v * g[t].double()).sum())
            total += float((v * gf[s].double()).sum())
        return total

    r = tfg.tfg_gated_recurrence(z.float(), x.float(), off, kind, initial=init.float())
    grads = tfg.tfg_gated_recurrence_backward(z.float(), x.float(), off, r.checkpoints, g, kind, initial=init.float(), grad_final=gf)
    at = [z, x, init]
    for i, grad in enumerate(grads):
        u = normal(*at[i].shape, 9 + i).double()
        plus, minus = ([v + s * 1e-4 * u if j == i else v for j, v in enumerate(at)] for s in (1, -1))
        slope = (loss(*plus) - loss(*minus)) / 2e-4
        assert abs(slope - float((grad.double() * u).sum())) <= 1e-5 * float(grad.double().norm() * u.norm())


def test_refusals():
    z, x = batch(20, 8, "sigmoid", "f32", 1)
    off = torch.tensor([0, 20], device="cuda")
    for bad in (dict(gate=z.t()), dict(x=x[:10]), dict(x=x.bfloat16()), dict(gate=z.half()), dict(node_offsets=off.int()),
                dict(kind="relu"), dict(initial=normal(2, 8, 1)), dict(gate=z[:, :1].expand(20, 8)), dict(gate=z.cpu())):
        with pytest.raises(ValueError):
            tfg.tfg_gated_recurrence(**{**dict(gate=z, x=x, node_offsets=off), **bad})
    with pytest.raises(tfg.TfgError):
        tfg.tfg_gated_recurrence(z, x, off, out=x)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_gated_recurrence(z.repeat(10, 1), x.repeat(10, 1), off, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    r = tfg.tfg_gated_recurrence(z, x, off, want_checkpoints=False, want_final=False)
    assert r.final is None
    with pytest.raises(ValueError):
        tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, x)
    with pytest.raises(ValueError):
        tfg.tfg_gated_recurrence_backward(z, x, off, normal(3, 8, 1), x)
    with pytest.raises(tfg.TfgError):
        tfg.tfg_gated_recurrence_backward(z, x, off, normal(1, 8, 1), x, grad_x=x)
