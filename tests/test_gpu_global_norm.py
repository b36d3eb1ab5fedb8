"""The global norm over many tensors and clipping by it, against 64-bit sums.

Tolerances, u = 2^-24: a thread's 32 squares are four fp32 chains of eight and two sums (10
roundings of positive terms), and everything after that keeps its rounding errors or is
fp64, so the sum of squares is off by 11 u at most and the norm by 5.5 u and its own
rounding: 7 u.  A clipped value has the factor's error (7 u and a rounding) and its
product's: 10 u, and half a step of bf16 (2^-8) where it is stored so.  Below 2^-126 the steps
of fp32 do not shrink with the value: half a step is 2^-150 for the norm, and as much for a
clipped value, whose bound has room for a few more (TINY).
"""
import math

import numpy as np
import pytest
import torch

from paper_2101_11552_gb300 import tfg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -150


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2101_11552_gb300 import build
    build.build_library()


def exact_norm(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


def check(tensors, clip, outs=None, inputs=None):
    inputs = inputs or [t.clone() for t in tensors]
    want = exact_norm(inputs)
    outs, norm = tfg.tfg_clip_by_global_norm(tensors, clip, outs=outs)
    assert abs(float(norm) - want) <= 7 * U * want + TINY
    assert float(tfg.tfg_global_norm(inputs)) == float(norm)
    factor = float(np.float32(clip)) / max(want, float(np.float32(clip)))
    for x, o in zip(inputs, outs):
        assert o.dtype == x.dtype and o.shape == x.shape
        w = x.double() * factor
        tol = (10 * U + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0)) * w.abs() + 4 * TINY
        assert bool(((o.double() - w).abs() <= tol).all())
    return outs, norm


SIZES = [[1], [0, 5, 0], [7, 64, 1000], [4096, 16384, 16385], [100_003, 41, 128 * 64, 1], [3] * 33, [70, 0, 1] * 200,
         [2_000_003, 5, 300_000], [1] * 1100]


@pytest.mark.parametrize("sizes", SIZES, ids=[f"{len(s)}x{max(s)}" for s in SIZES])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
def test_norm_and_clip(sizes, kind):
    gen = torch.Generator(device="cuda").manual_seed(sum(sizes))
    types = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.bfloat16, torch.float32]}[kind]
    ts = [torch.randn(k, device="cuda", generator=gen, dtype=types[i % len(types)]) for i, k in enumerate(sizes)]
    norm = exact_norm(ts)
    check(ts, 0.25 * norm)
    outs, _ = check(ts, 4.0 * norm)
    for a, b in zip(ts, outs):
        assert torch.equal(a, b) and (a.numel() == 0 or a.data_ptr() != b.data_ptr())


def test_in_place_and_into_buffers():
    gen = torch.Generator(device="cuda").manual_seed(3)
    flat = torch.randn(50_000, device="cuda", generator=gen)
    # pieces of one buffer, off the 16-byte boundary, in place
    cuts = [0, 1, 4, 1000, 1003, 33_333, 50_000]
    ts = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
    before = [t.clone() for t in ts]
    outs, _ = check(ts, 1.0, outs=ts, inputs=before)
    assert all(a.data_ptr() == b.data_ptr() for a, b in zip(ts, outs))
    # a second time: the norm is 1 within rounding, values move by rounding alone
    after = [t.clone() for t in ts]
    check(ts, 1.0, outs=ts, inputs=after)
    for dt in (torch.float32, torch.bfloat16):
        x = [torch.randn(k, device="cuda", generator=gen).to(dt) for k in (999, 8, 20_000)]
        buf = torch.zeros(30_000, device="cuda", dtype=dt)
        to = [buf[1:1000], buf[1001:1009], buf[1010:21_010]]              # unaligned outputs
        check(x, 0.5, outs=to)
        assert float(buf[0]) == 0 and float(buf[1000]) == 0 and float(buf[1009]) == 0 and bool((buf[21_010:] == 0).all())


def test_rows_of_a_matrix_are_not_read_as_one():
    m = torch.randn(10, 7, device="cuda")
    with pytest.raises(ValueError):
        tfg.tfg_global_norm([m[:, :3]])
    with pytest.raises(ValueError):
        tfg.tfg_global_norm([m.half()])
    with pytest.raises(ValueError):
        tfg.tfg_clip_by_global_norm([m], 1.0, outs=[m.view(-1)[:69]])
    for outs in ([m, m], [m.view(-1)[:35], m.view(-1)[34:69]]):
        with pytest.raises(tfg.TfgError) as e:
            tfg.tfg_clip_by_global_norm([m, m] if outs[0] is m else [m.view(-1)[:35].clone(), m.view(-1)[:35].clone()],
                                        1.0, outs=outs)
        assert e.value.code == tfg.TFG_ERR_INVALID_ARG


def test_no_values():
    assert float(tfg.tfg_global_norm([])) == 0
    outs, norm = tfg.tfg_clip_by_global_norm([], 1.0)
    assert outs == [] and float(norm) == 0
    e = torch.empty(0, device="cuda")
    outs, norm = tfg.tfg_clip_by_global_norm([e, e.bfloat16()], 1.0)
    assert float(norm) == 0
    outs, norm = tfg.tfg_clip_by_global_norm([torch.zeros(70_000, device="cuda")], 1.0)
    assert float(norm) == 0 and bool((outs[0] == 0).all())


@pytest.mark.parametrize("size", [1e-40, 1e-30, 3e-23, 1e-12, 1.0, 1e15, 1e19, 1e30])
@pytest.mark.parametrize("n", [1, 31, 5000, 100_000])
def test_squares_outside_fp32(size, n):
    """Values whose squares leave the range of fp32 at either end, among zeros and others."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, device="cuda", generator=gen) * size
    zeros = torch.zeros(40_000, device="cuda")
    outs, _ = check([x, zeros], 0.5 * float(np.float32(min(exact_norm([x]), 3e38))) or 1e-38)
    mixed = torch.cat([x, torch.full((64,), 1e-25, device="cuda"), torch.full((3,), 1e17, device="cuda"), zeros])
    check([mixed], 2.0)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_not_finite(bad):
    ts = [torch.randn(5000, device="cuda"), torch.randn(300, device="cuda", dtype=torch.bfloat16)]
    ts[1][77] = bad
    outs, norm = tfg.tfg_clip_by_global_norm(ts, 1.0)
    assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(bad)
    assert all(bool(torch.isnan(o.float()).all()) for o in outs)
    outs, norm = tfg.tfg_clip_by_global_norm([torch.full((100,), 1e38, device="cuda")], 1.0)   # the norm passes fp32
    assert math.isinf(float(norm)) and bool(torch.isnan(outs[0]).all())


def test_captured_and_on_another_stream():
    ts = [torch.randn(k, device="cuda") for k in (1000, 7, 40_000)]
    outs = [torch.empty_like(t) for t in ts]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tfg.tfg_clip_by_global_norm(ts, 1.0, outs=outs)
    side.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    ws = torch.empty(tfg.tfg_global_norm_workspace_size(3), dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(graph):
        _, norm = tfg.tfg_clip_by_global_norm(ts, 1.0, outs=outs, workspace=ws)
    with torch.cuda.graph(second):                                        # two captured calls share a workspace
        _, small = tfg.tfg_clip_by_global_norm(ts[1:2], 0.5, outs=ts[1:2], workspace=ws)
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in ts:
            t.normal_(generator=g)
        want = exact_norm(ts)
        own = exact_norm(ts[1:2])
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        assert abs(float(norm) - want) <= 7 * U * want and abs(float(small) - own) <= 7 * U * own
        assert abs(exact_norm(outs) - 1.0) <= 20 * U and abs(exact_norm(ts[1:2]) - 0.5) <= 20 * U


def test_more_than_2_32_values():
    n = (1 << 32) + 12_345
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    x[-1] = 3.0
    want = math.sqrt(n + 8)
    outs, norm = tfg.tfg_clip_by_global_norm([x, torch.ones(5, device="cuda")], 65536.0, outs=[x, torch.empty(5, device="cuda")])
    want = math.sqrt(n + 8 + 5)
    assert abs(float(norm) - want) <= 7 * U * want
    f = 65536.0 / want
    assert bool((x[:-1] == x[0]).all()) and abs(float(x[0]) - f) <= 2.0 ** -8 * f and abs(float(x[-1]) - 3 * f) <= 2.0 ** -8 * 3 * f


@pytest.mark.parametrize("size,clip", [(1e36, 1e-3), (1e36, 1e-6), (3e35, 1e-9), (1e20, 1e-20), (1e30, 1e-30)])
def test_factors_below_the_normal_numbers(size, clip):
    """clip_norm / norm has no fp32 value of full precision; the clipped values have."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    ts = [torch.randn(k, device="cuda", generator=gen, dtype=dt) * size
          for k, dt in ((5000, torch.float32), (999, torch.bfloat16), (1, torch.float32))]
    outs, _ = check(ts, clip)
    assert float(outs[0].abs().max()) > clip * 1e-2
    before = [t.clone() for t in ts]
    check(ts, clip, outs=ts, inputs=before)
