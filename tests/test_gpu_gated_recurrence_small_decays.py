"""Gated recurrence where gates forget strongly: a far below 1 keeps its own digits, forward and in every gradient.

Bounds as in test_gpu_gated_recurrence.py, u = 2^-24, but every error of a gate is relative to what it is an error of.
With the sigmoid gate a is e / (1 + e), e = e^z, for z < 0: z log2 e and its constant are rounded (2 |z| u of e), the exponential
and the reciprocal are within 2 units of the last place (4 u), a sum and a product are rounded: ea = (2 |z| + 10) u a, and
1 - a then has ep = ea + u p.  For z >= 0 it is p = 1 - a that is formed so, ep = (2 a |z| + 7) u p, and a v is taken as
v + (a - 1) v: ea = ep.  From -5.55 to 0 a may be taken so too: e is off by (2 |z| + 4) u of itself, the sum and the reciprocal by 3 u p,
3 u p more in ea.  With the exp gate ea = (2 |z| + 6) u a away from 0 (the exponential and a rounding), and from -0.35 to 0
p = a - 1 has 2 u: ea = 5 u |p|.  Hence
  E_t = a_t E_{t-1} + ea M_{t-1} + ep |x_t| + 8 u M_t,     M_t = a_t M_{t-1} + |b_t|     (exp gate: b = x, exact)
  F_t = (a F + ea L)_{t+1} + 8 u L_t,                      L_t = |g_t| + a_{t+1} L_{t+1}
  grad_x:       F p + L (ep + 2 u p)                                                     (exp gate: F)
  grad_gate:    with W = M_{t-1} + |x_t|: a p (F W + L E_{t-1}) + L W (p ea + a ep + 6 u a p)    (exp gate: a F M + a L E + L M (ea + 4 u a))
  grad_initial: a F + L (ea + 2 u a)
A state composed over a thread's rows or more costs what its rows cost, and less than 8 u.  a below 2^-126 is 0: 2^-126 in ea, and a
term of 1e-40 for values below the normal numbers.
"""
import pytest
import torch

from paper_2101_11552_gb300 import tfg
from test_gpu_gated_recurrence import U, _built, close, normal  # noqa: F401

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TINY = 2.0 ** -126


def gates(z, kind):
    """a, 1 - a (exp: a - 1), and their errors."""
    z = z.double().cpu()
    far = z.abs().clamp(max=200)
    if kind == "exp":
        a, p = torch.exp(z), torch.expm1(z)
        return a, p, torch.where((z >= -0.35) & (z < 0), 5 * U * p.abs(), (2 * far + 6) * U * a) + TINY, torch.zeros_like(a)
    a, p = torch.sigmoid(z), torch.sigmoid(-z)
    ea, ep = (2 * far + 10) * U * a + TINY + torch.where(z >= -5.55, 3 * U * p, 0.0), (2 * a * far + 7) * U * p + TINY
    return a, p, torch.where(z < 0, ea, ep), torch.where(z < 0, ea + U * p, ep)


def check(z, x, offsets, kind, initial, g, grad_final=None):
    """One call of each direction against the 64-bit recurrence."""
    off = torch.tensor(offsets, device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off, kind, initial=initial, out_dtype=torch.float32)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, initial=initial, grad_final=grad_final)
    a, p, ea, ep = gates(z, kind)
    n, f = a.shape
    x, g = x.double().cpu(), g.double().cpu()
    state = initial.double().cpu()
    last = torch.zeros_like(state) if grad_final is None else grad_final.double().cpu()
    sigmoid = kind == "sigmoid"
    add, bx = (p * x, x.abs()) if sigmoid else (x, torch.zeros_like(x))
    v, e, before, m_before, e_before, lam, size, err = (torch.zeros(n, f, dtype=torch.float64) for _ in range(8))
    first, first_tol, final, final_tol = (torch.zeros_like(state) for _ in range(4))
    for s, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        vt, mt, et = state[s], state[s].abs(), torch.zeros(f, dtype=torch.float64)
        for t in range(lo, hi):
            before[t], m_before[t], e_before[t] = vt, mt, et
            et = a[t] * et + ea[t] * mt + ep[t] * bx[t]
            vt, mt = a[t] * vt + add[t], a[t] * mt + add[t].abs()
            et = et + 8 * U * mt
            v[t], e[t] = vt, et
        final[s], final_tol[s] = vt, et
        c, l, ft = last[s], last[s].abs(), torch.zeros(f, dtype=torch.float64)
        for t in range(hi - 1, lo - 1, -1):
            lam[t], size[t] = g[t] + c, g[t].abs() + l
            err[t] = ft + 8 * U * size[t]
            c, l, ft = a[t] * lam[t], a[t] * size[t], a[t] * err[t] + ea[t] * size[t]
        first[s], first_tol[s] = c, ft + 2 * U * a[lo] * size[lo]
    close(r.out, v, e, "out")
    close(r.final, final, final_tol, "final")
    if sigmoid:
        gx, gx_tol = lam * p, err * p + size * (ep + 2 * U * p)
        way = m_before + bx
        gz = lam * (before - x) * a * p
        gz_tol = a * p * (err * way + size * e_before) + size * way * (p * ea + a * ep + 6 * U * a * p)
    else:
        gx, gx_tol = lam, err
        gz = lam * before * a
        gz_tol = a * (err * m_before + size * e_before) + size * m_before * (ea + 4 * U * a)
    close(b.gate, gz, gz_tol, "grad_gate")
    close(b.x, gx, gx_tol, "grad_x")
    close(b.initial, first, first_tol, "grad_initial")
    return r, b


KINDS = ["sigmoid", "exp"]
WIDTHS = [(64, "f32"), (33, "f32"), (72, "bf16"), (21, "bf16")]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f,dt", WIDTHS)
@pytest.mark.parametrize("input", ["none", "some"])
def test_one_row_from_a_large_state(input, f, dt, kind):
    """Gates from -85 to 0, states of 1e10: what is left of them, and the gates' gradients."""
    n = 300
    z = torch.linspace(-85, 0, n * f, device="cuda").view(f, n).t().contiguous().to(DT[dt])
    x = (normal(n, f, 1) if input == "some" else torch.zeros(n, f, device="cuda")).to(DT[dt])
    check(z, x, list(range(n + 1)), kind, normal(n, f, 2) * 1e10, normal(n, f, 3), normal(n, f, 4))


def test_the_values_at_the_gates_where_nothing_was_left():
    """z = -18, a state of 1e10: 152.3 and not 0; slopes at -16, -17, -20."""
    z = torch.tensor([[-18.0, -16.0, -17.0, -20.0]], device="cuda")
    x, off, init = torch.zeros(1, 4, device="cuda"), torch.tensor([0, 1], device="cuda"), torch.full((1, 4), 1e10, device="cuda")
    for kind in KINDS:
        a = torch.exp(z.double()) if kind == "exp" else torch.sigmoid(z.double())
        r = tfg.tfg_gated_recurrence(z, x, off, kind, initial=init)
        assert torch.allclose(r.out.double(), 1e10 * a, rtol=(2 * 20 + 20) * U, atol=0)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, torch.ones_like(x), kind, initial=init)
        slope = a if kind == "exp" else a * (1 - a)
        assert torch.allclose(b.gate.double(), 1e10 * slope, rtol=(2 * 20 + 30) * U, atol=0)
        assert torch.allclose(b.initial.double(), a, rtol=(2 * 20 + 20) * U, atol=0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f,dt", WIDTHS)
@pytest.mark.parametrize("input", [0.0, 1e-6])
def test_cuts_along_a_sequence(input, f, dt, kind):
    """A large state that is cut down at a few rows, in tiles and at their borders, and kept in between."""
    n, offsets = 700, [0, 420, 700]
    gen = torch.Generator(device="cuda").manual_seed(f)
    z = torch.full((n, f), 12.0 if kind == "sigmoid" else -2.0 ** -17, device="cuda")
    for t in (3, 64, 127, 128, 300, 383, 420, 511, 640, 699):
        z[t] = -9.0 - 3.0 * torch.rand(f, device="cuda", generator=gen)
    x = input * torch.randn(n, f, device="cuda", generator=gen)
    check(z.to(DT[dt]), x.to(DT[dt]), offsets, kind, 1e15 * normal(2, f, 2), normal(n, f, 3), normal(2, f, 4))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f,dt", WIDTHS)
def test_gates_of_all_sizes(f, dt, kind):
    """Both forms of a word side by side in a row, and at the borders between them."""
    n, offsets = 600, [0, 1, 129, 450, 600]
    gen = torch.Generator(device="cuda").manual_seed(f + 1)
    z = 4.0 * torch.randn(n, f, device="cuda", generator=gen)
    if kind == "exp":
        z = -z.abs() * (torch.rand(n, f, device="cuda", generator=gen) < 0.5) * 0.25
    edge = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.35, -0.35, 0.3501, -0.3501, -5.55, -1e-7], device="cuda")
    z[:, 5] = edge.repeat(n // 10)
    check(z.to(DT[dt]), normal(n, f, 5).to(DT[dt]), offsets, kind, normal(4, f, 2), normal(n, f, 3), normal(4, f, 4))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("f,dt", [(16, "f32"), (7, "f32"), (16, "bf16")])
def test_a_long_memory_has_no_drift(f, dt, kind):
    """Errors of a memory of L rows, as a share of the values' norm.  Gates that differ from row to row: the roundings of
    states and of products of decays go up as often as down and come to less than u sqrt(L), 100 u for 10,000 rows; what is
    wrong in every decay the same way comes to L times as much: half a u in each (an exponential's last bits) to 5,000 u.
    300 u where two such errors meet.  (Under one gate throughout, a product is rounded the same way every time, too.)"""
    n = 40_000
    reach = torch.logspace(1.5, 4, f, dtype=torch.float64)                 # rows
    spread = torch.exp(0.5 * normal(n, f, 3))
    z = -spread / reach.float().cuda() if kind == "exp" else torch.log(reach.float().cuda() * spread)
    z = z.to(DT[dt])
    x, g, off = normal(n, f, 1).to(DT[dt]), normal(n, f, 2), torch.tensor([0, n], device="cuda")
    r = tfg.tfg_gated_recurrence(z, x, off, kind, out_dtype=torch.float32)
    b = tfg.tfg_gated_recurrence_backward(z, x, off, r.checkpoints, g, kind, initial=torch.zeros(1, f, device="cuda"))
    a, p, _, _ = gates(z, kind)
    xs, gs = x.double().cpu(), g.double().cpu()
    add = p * xs if kind == "sigmoid" else xs
    v, lam = torch.zeros(n, f, dtype=torch.float64), torch.zeros(n, f, dtype=torch.float64)
    state = torch.zeros(f, dtype=torch.float64)
    for t in range(n):
        state = a[t] * state + add[t]
        v[t] = state
    carry = torch.zeros(f, dtype=torch.float64)
    for t in range(n - 1, -1, -1):
        lam[t] = gs[t] + carry
        carry = a[t] * lam[t]
    before = torch.cat([torch.zeros(1, f, dtype=torch.float64), v[:-1]])
    gz = lam * (before - xs) * a * p if kind == "sigmoid" else lam * before * a
    step = 0.0 if dt == "f32" else 2.0 ** -8
    for got, want, tol in ((r.out, v, 100 * U), (b.x, lam * p if kind == "sigmoid" else lam, 100 * U + step), (b.gate, gz, 300 * U + step)):
        off_by = (got.double().cpu() - want).norm(dim=0) / want.norm(dim=0)
        assert bool((off_by <= tol).all()), off_by
