"""Embedding lookup, grouping of ids and the table's gradient against plain 64-bit forms.

Tolerances, u = 2^-24:
  * lookup: one fp32 product (u), and for a bf16 result one more rounding of at most half a
    step (2^-8), each relative to the value;
  * gradient: a row that m positions name is a sum of m fp32 terms in some fixed order, off
    by at most m u times the sum of their absolute values to first order, and one product;
    (m + 4) u of scale * sum |g| covers it with the second-order terms (m u < 1e-2 here).
"""
import numpy as np
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


def make_ids(n, rows, kind, pad, rng):
    if kind == "one":
        ids = np.full(n, rows // 2, np.int64)
    elif kind == "skew":
        ids = np.minimum((rows * rng.random(n) ** 6).astype(np.int64), rows - 1)
    else:
        ids = rng.integers(0, rows, n)
    if pad is not None:
        ids[rng.random(n) < 0.2] = pad
    return ids.astype(np.int64)


def check_lookup(table, ids, scale, pad, out):
    t = table.double().cpu()
    ids = torch.as_tensor(ids)
    want = torch.zeros(ids.numel(), t.shape[1], dtype=torch.float64)
    here = torch.ones_like(ids, dtype=torch.bool) if pad is None else ids != pad
    want[here] = t[ids[here]] * float(np.float32(scale))
    tol = (2 * U + (2.0 ** -8 if out.dtype == torch.bfloat16 else 0.0)) * want.abs()
    off = (out.double().cpu().reshape(want.shape) - want).abs()
    assert bool((off <= tol).all()), f"worst excess {(off - tol).max()}"
    assert bool((out.reshape(want.shape)[~here.cuda()] == 0).all())


def check_groups(groups, ids, rows, pad):
    key = np.where(ids == pad, rows, ids) if pad is not None else ids
    order = np.argsort(key, kind="stable")
    assert np.array_equal(groups.perm.cpu().numpy(), order)
    assert np.array_equal(groups.sorted_ids.cpu().numpy(), key[order])
    assert np.array_equal(groups.rowptr.cpu().numpy(), np.searchsorted(key[order], np.arange(rows + 1)))
    tfg.check_status(groups.status)


def check_gradient(grad, ids, rows, pad, scale, got):
    g = grad.double().cpu().reshape(len(ids), -1)
    ids = torch.as_tensor(ids)
    here = torch.ones_like(ids, dtype=torch.bool) if pad is None else ids != pad
    s = float(np.float32(scale))
    want = torch.zeros(rows, g.shape[1], dtype=torch.float64).index_add_(0, ids[here], g[here]) * s
    size = torch.zeros(rows, g.shape[1], dtype=torch.float64).index_add_(0, ids[here], g[here].abs()) * abs(s)
    m = torch.bincount(ids[here], minlength=rows).double()[:, None]
    off = (got.double().cpu() - want).abs()
    assert bool((off <= (m + 4) * U * size).all()), f"worst {(off / size.clamp(min=1e-300)).max()}"


@pytest.mark.parametrize("n,rows,f,kind,pad", [
    (1, 1, 1, "uniform", None), (1, 7, 4, "uniform", None), (2, 3, 5, "one", None), (31, 4, 8, "uniform", -1),
    (33, 100, 3, "skew", 0), (257, 5, 16, "one", -1), (1000, 119, 128, "skew", None), (2048, 50, 17, "uniform", 49),
    (2049, 3000, 41, "skew", -7), (4097, 2, 100, "one", None), (5000, 20000, 132, "uniform", -1),
    (20000, 119, 64, "skew", None), (20011, 119, 123, "one", 3), (131073, 119, 8, "skew", None),
    (140000, 1000, 12, "one", None), (30000, 700, 300, "skew", None), (9000, 5, 520, "skew", -1)])
@pytest.mark.parametrize("table_t,out_t,id_t", [("f32", "f32", torch.int64), ("bf16", "bf16", torch.int32),
                                                ("f32", "bf16", torch.int32), ("bf16", "f32", torch.int64)])
def test_lookup_groups_and_gradient(n, rows, f, kind, pad, table_t, out_t, id_t):
    rng = np.random.default_rng(n + 31 * rows + f)
    ids = make_ids(n, rows, kind, pad, rng)
    gen = torch.Generator(device="cuda").manual_seed(n + f)
    table = torch.randn(rows, f, device="cuda", generator=gen, dtype=DT[table_t])
    grad = torch.randn(n, f, device="cuda", generator=gen, dtype=DT[out_t])
    scale = float(np.sqrt(f))
    dids = torch.as_tensor(ids).to(id_t).cuda()
    out, status = tfg.tfg_embedding_lookup(table, dids, scale, padding_id=pad, out_dtype=DT[out_t])
    tfg.check_status(status)
    assert out.dtype == DT[out_t] and out.shape == (n, f)
    check_lookup(table, ids, scale, pad, out)
    groups = tfg.tfg_group_ids(dids, rows, padding_id=pad)
    check_groups(groups, ids, rows, pad)
    got = tfg.tfg_embedding_backward(groups, grad, scale)
    check_gradient(grad, ids, rows, pad, scale, got)
    again = tfg.tfg_embedding_backward(tfg.tfg_group_ids(dids, rows, padding_id=pad), grad, scale)
    assert torch.equal(got, again)


@pytest.mark.parametrize("n", [1, 2, 700, 2047, 2048, 2049, 8191, 16384, 16385, 32769, 65536, 65537, 100_001, 131_072, 131_073, 400_000])
@pytest.mark.parametrize("rows,kind", [(3, "uniform"), (511, "skew"), (512, "one"), (4095, "uniform"), (4096, "uniform"), (40_000, "uniform"), (300_000, "skew")])
def test_grouping_sizes(n, rows, kind):
    """One CTA and many, counts added up by the downsweep or scanned, one to three digits."""
    ids = make_ids(n, rows, kind, -1, np.random.default_rng(n + rows))
    check_groups(tfg.tfg_group_ids(torch.as_tensor(ids).cuda(), rows, padding_id=-1), ids, rows, -1)


def test_many_passes_of_the_sort():
    """Tables of more than 2^18 rows take three digits; counters over more than 64 tiles the
    scan kernel."""
    rng = np.random.default_rng(5)
    for rows, n in [(300_001, 5000), (1 << 27, 3000), (600_000, 200_000)]:
        ids = make_ids(n, rows, "uniform", -1, rng)
        ids[:3] = [0, rows - 1, rows // 2]
        groups = tfg.tfg_group_ids(torch.as_tensor(ids).cuda(), rows, padding_id=-1)
        check_groups(groups, ids, rows, -1)


@pytest.mark.parametrize("f", [8, 100, 33])
def test_misaligned_and_shaped(f):
    """Pointers off the 16-byte boundary take the scalar kernels; ids of any shape."""
    rng = np.random.default_rng(f)
    rows, shape = 40, (13, 29)
    ids = rng.integers(0, rows, shape)
    n = ids.size
    for dt in (torch.float32, torch.bfloat16):
        table = torch.randn(rows * f + 1, device="cuda").to(dt)[1:].view(rows, f)
        grad = torch.randn(n * f + 3, device="cuda").to(dt)[3:].view(*shape, f)
        dids = torch.as_tensor(ids).cuda()
        out = torch.empty(n * f + 1, device="cuda", dtype=dt)[1:].view(*shape, f)
        got, status = tfg.tfg_embedding_lookup(table, dids, 0.5, out=out)
        tfg.check_status(status)
        assert got.data_ptr() == out.data_ptr()
        check_lookup(table, ids.reshape(-1), 0.5, None, out)
        groups = tfg.tfg_group_ids(dids, rows)
        to = torch.empty(rows * f + 1, device="cuda")[1:].view(rows, f)
        check_gradient(grad, ids.reshape(-1), rows, None, 0.5, tfg.tfg_embedding_backward(groups, grad, 0.5, out=to))


def test_empty_inputs():
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    table = torch.randn(5, 4, device="cuda")
    out, status = tfg.tfg_embedding_lookup(table, none)
    tfg.check_status(status)
    assert out.shape == (0, 4)
    groups = tfg.tfg_group_ids(none, 5)
    assert groups.rowptr.cpu().tolist() == [0] * 6
    tfg.check_status(groups.status)
    assert bool((tfg.tfg_embedding_backward(groups, torch.empty(0, 4, device="cuda")) == 0).all())
    # a table without rows: every position is padding
    ids = torch.full((3,), -1, dtype=torch.int64, device="cuda")
    out, status = tfg.tfg_embedding_lookup(torch.empty(0, 4, device="cuda"), ids, padding_id=-1)
    tfg.check_status(status)
    assert bool((out == 0).all())
    groups = tfg.tfg_group_ids(ids, 0, padding_id=-1)
    assert groups.rowptr.cpu().tolist() == [0] and groups.perm.cpu().tolist() == [0, 1, 2]
    assert tfg.tfg_embedding_backward(groups, torch.ones(3, 4, device="cuda")).shape == (0, 4)
    # padding alone
    ids = torch.full((500,), 2, dtype=torch.int32, device="cuda")
    groups = tfg.tfg_group_ids(ids, 5, padding_id=2)
    assert groups.rowptr.cpu().tolist() == [0] * 6
    assert bool((tfg.tfg_embedding_backward(groups, torch.ones(500, 4, device="cuda")) == 0).all())


def test_ids_outside_the_table_are_reported_and_stand_for_no_row():
    table = torch.randn(10, 6, device="cuda")
    for bad in (10, -1, 2**31 - 1, -2**31):
        ids = torch.tensor([1, bad, 3], dtype=torch.int64, device="cuda")
        out, status = tfg.tfg_embedding_lookup(table, ids)
        assert int(status) == tfg.TFG_ERR_INDEX_RANGE
        assert bool((out[1] == 0).all())
        groups = tfg.tfg_group_ids(ids, 10)
        assert int(groups.status) == tfg.TFG_ERR_INDEX_RANGE
        assert groups.perm.cpu().tolist() == [0, 2, 1]
    out, status = tfg.tfg_embedding_lookup(table, ids[:1])                # the next call reports nothing
    tfg.check_status(status)


def test_not_finite_gradients_stay_in_their_rows():
    rng = np.random.default_rng(0)
    ids = make_ids(3000, 50, "skew", -1, rng)
    at = int(np.flatnonzero(ids == 7)[0]) if (ids == 7).any() else 0
    ids[at] = 7
    grad = torch.ones(3000, 36, device="cuda")
    grad[at, 5], grad[int(np.flatnonzero(ids == -1)[0])] = float("inf"), float("nan")
    got = tfg.tfg_embedding_backward(tfg.tfg_group_ids(torch.as_tensor(ids).cuda(), 50, padding_id=-1), grad)
    bad = ~torch.isfinite(got)
    assert bad.sum() == 1 and bool(bad[7, 5])


def test_captured_and_on_another_stream():
    rows, n, f = 119, 4000, 48
    ids = torch.randint(0, rows, (n,), device="cuda")
    table, grad = torch.randn(rows, f, device="cuda"), torch.randn(n, f, device="cuda")

    def step():
        out, _ = tfg.tfg_embedding_lookup(table, ids, 2.0)
        return out, tfg.tfg_embedding_backward(tfg.tfg_group_ids(ids, rows), grad, 2.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, gt = step()
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        ids.copy_(torch.randint(0, rows, (n,), device="cuda", generator=g))
        grad.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        check_lookup(table, ids.cpu().numpy(), 2.0, None, out)
        check_gradient(grad, ids.cpu().numpy(), rows, None, 2.0, gt)


def test_more_than_2_31_elements():
    """Row offsets past 32 bits in the table, the output and the gradient (bf16)."""
    rows, f, n = 17_000_001, 130, 17_200_003
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn(rows, f, device="cuda", generator=gen, dtype=torch.bfloat16)
    ids = torch.randint(0, rows, (n,), device="cuda", generator=gen)
    ids[-1], ids[-2], ids[0] = rows - 1, 0, rows - 1
    out, status = tfg.tfg_embedding_lookup(table, ids)
    tfg.check_status(status)
    look = torch.cat([torch.arange(1000, device="cuda"), torch.arange(n - 1000, n, device="cuda")])
    assert torch.equal(out[look], table[ids[look]])
    groups = tfg.tfg_group_ids(ids, rows)
    tfg.check_status(groups.status)
    got = tfg.tfg_embedding_backward(groups, out)
    for v in (0, rows - 1, int(ids[n // 2]), int(ids[n - 5])):
        at = torch.nonzero(ids == v).flatten()
        want = out[at].double().sum(0)
        assert bool(((got[v].double() - want).abs() <= (len(at) + 4) * U * out[at].double().abs().sum(0)).all())
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[ids] = True
    assert bool((got[~named] == 0).all())


def test_binding_refuses():
    table, ids = torch.randn(5, 4, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        tfg.tfg_embedding_lookup(table, ids.short())
    with pytest.raises(ValueError):
        tfg.tfg_embedding_lookup(table.t(), ids)                           # not contiguous
    with pytest.raises(ValueError):
        tfg.tfg_embedding_lookup(table.half(), ids)
    with pytest.raises(ValueError):
        tfg.tfg_embedding_lookup(table, ids, out=torch.empty(4, 4, device="cuda"))
    groups = tfg.tfg_group_ids(ids, 5)
    with pytest.raises(ValueError):
        tfg.tfg_embedding_backward(groups, torch.randn(4, 4, device="cuda"))
    with pytest.raises(tfg.TfgError) as e:
        tfg.tfg_group_ids(ids.repeat(1000), 5, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.code == tfg.TFG_ERR_WORKSPACE


@pytest.mark.parametrize("bad", [2 ** 63, 2 ** 64 - 1, 2 ** 64 + 2, -2 ** 63 - 1])
def test_padding_ids_that_no_int64_holds_are_refused(bad):
    """They would be taken for the id that they equal in the lowest 64 bits."""
    table, ids = torch.randn(5, 4, device="cuda"), torch.tensor([0, 2, -1], device="cuda")
    with pytest.raises(ValueError):
        tfg.tfg_embedding_lookup(table, ids, padding_id=bad)
    with pytest.raises(ValueError):
        tfg.tfg_group_ids(ids, 5, padding_id=bad)
