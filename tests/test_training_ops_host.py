"""Refusals of the embedding, group-norm and clipping entry points: every bad argument is
rejected on the host before anything is enqueued (no GPU needed)."""
import ctypes
import math

import pytest

FAKE = ctypes.c_void_p(0x100000)         # never dereferenced: every call below fails validation
OTHER = ctypes.c_void_p(0x900000)
OUT = ctypes.c_void_p(0x40000000)
WS = ctypes.c_void_p(0x80000000)


@pytest.fixture(scope="module")
def lib():
    from paper_2101_11552_gb300 import build, tfg
    build.build_library()
    return tfg.lib()


def caller(fn, defaults):
    def call(**kw):
        assert set(kw) <= set(defaults), kw
        return fn(*[kw.get(k, v) for k, v in defaults.items()])
    return call


def err(lib):
    return lib.tfg_last_error().decode()


@pytest.mark.parametrize("name", ["tfg_embedding_lookup", "tfg_embedding_lookup32"])
def test_lookup_rejects(lib, name):
    call = caller(getattr(lib, name), dict(ids=FAKE, n=10, table=OTHER, tdt=0, rows=7, f=4, scale=1.0, pad=-1, out=OUT,
                                           odt=0, status=FAKE, st=None))
    assert call(n=-1) == -1 and call(rows=-1) == -1 and call(f=0) == -1
    assert call(n=2**31 - 1) == -2 and call(rows=2**31 - 1) == -2
    assert call(f=65535 * 128 + 1) == -2 and "features" in err(lib)
    assert call(tdt=2) == -1 and call(odt=-1) == -1
    assert call(ids=None) == -1 and "ids" in err(lib)
    assert call(table=None) == -1 and call(out=None) == -1 and call(status=None) == -1
    assert call(out=OTHER) == -1 and "overlap" in err(lib)
    assert call(out=ctypes.c_void_p(0x900000 + 7 * 4 * 4 - 4)) == -1       # the table's last value
    assert call(out=FAKE) == -1                                             # the ids
    assert call(table=ctypes.c_void_p(0x900002)) == -1 and "aligned" in err(lib)
    assert call(out=ctypes.c_void_p(0x40000001), odt=1) == -1


@pytest.mark.parametrize("name", ["tfg_group_ids", "tfg_group_ids32"])
def test_group_ids_rejects(lib, name):
    call = caller(getattr(lib, name), dict(ids=FAKE, n=10, rows=7, pad=-1, rowptr=OUT, sorted=OUT, perm=OUT, ws=WS,
                                           wsb=1 << 20, status=FAKE, st=None))
    assert call(n=-1) == -1 and call(rows=-1) == -1
    assert call(n=2**31 - 1) == -2
    for missing in ("ids", "rowptr", "sorted", "perm", "status"):
        assert call(**{missing: None}) == -1, missing
    assert call(n=5000, ws=None) == -3 and call(n=5000, wsb=16) == -3 and "workspace" in err(lib)
    assert call(n=5000, ws=ctypes.c_void_p(0x80000010)) == -1


def test_group_ids_workspace(lib):
    n = ctypes.c_size_t(0)
    ws = lib.tfg_group_ids_workspace_size
    assert ws(119, 112640, ctypes.byref(n)) == 0 and n.value > 0
    one = n.value
    assert ws(50000, 112640, ctypes.byref(n)) == 0 and n.value >= one + 8 * 112640      # two passes: a pair buffer
    assert ws(50000, 2048, ctypes.byref(n)) == 0 and n.value == 0                       # one CTA
    assert ws(-1, 5, ctypes.byref(n)) == -1 and ws(5, 5, None) == -1 and ws(5, 2**31, ctypes.byref(n)) == -2


def test_embedding_backward_rejects(lib):
    call = caller(lib.tfg_embedding_backward, dict(rowptr=FAKE, sorted=FAKE, perm=FAKE, g=OTHER, gdt=0, n=10, rows=7, f=4,
                                                   scale=1.0, out=OUT, ws=WS, wsb=1 << 24, st=None))
    for missing in ("rowptr", "sorted", "perm", "g", "out"):
        assert call(**{missing: None}) == -1, missing
    assert call(ws=None) == -3 and call(wsb=1024) == -3 and call(ws=ctypes.c_void_p(0x80000008)) == -1
    assert call(gdt=3) == -1 and call(f=0) == -1 and call(n=-1) == -1 and call(rows=2**31) == -2
    assert call(out=OTHER) == -1 and "overlap" in err(lib)
    n = ctypes.c_size_t(0)
    assert lib.tfg_embedding_backward_workspace_size(128, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.tfg_embedding_backward_workspace_size(0, ctypes.byref(n)) == -1


NORM = dict(x=FAKE, xdt=0, off=OTHER, n=100, g=3, f=24, k=4, gamma=None, beta=None, eps=1e-5, act=1, out=OUT, odt=0,
            mean=None, rstd=None, ws=None, wsb=0, status=FAKE, st=None)


def test_group_norm_rejects(lib):
    call = caller(lib.tfg_group_norm, NORM)
    assert call(n=-1) == -1 and call(g=-1) == -1 and call(f=0) == -1
    assert call(n=2**31) == -2 and call(g=2**31) == -2
    assert call(k=0) == -1 and call(k=5) == -1 and "num_groups" in err(lib)
    assert call(f=2050, k=2) == -2 and "channels per group" in err(lib)
    assert call(xdt=7) == -1 and call(odt=7) == -1
    assert call(act=4) == -1 and call(act=-1) == -1 and "activation" in err(lib)
    for eps in (0.0, -1.0, math.inf, math.nan):
        assert call(eps=eps) == -1, eps
    for missing in ("x", "off", "out", "status"):
        assert call(**{missing: None}) == -1, missing
    assert call(mean=FAKE) == -1 and call(rstd=FAKE) == -1
    assert call(out=FAKE) == -1 and "overlap" in err(lib)
    assert call(x=ctypes.c_void_p(0x100002)) == -1 and call(out=ctypes.c_void_p(0x40000001), odt=1) == -1
    assert call(n=200000) == -3 and "workspace" in err(lib)              # graphs may be large: partial statistics
    assert call(n=200000, ws=ctypes.c_void_p(0x80000008), wsb=1 << 30) == -1
    assert call(n=2**31 - 1, g=2**31 - 1, f=4096, k=4096) == -2          # more teams than a grid holds


def test_group_norm_backward_rejects(lib):
    call = caller(lib.tfg_group_norm_backward, dict(
        x=FAKE, xdt=0, off=OTHER, n=100, g=3, f=24, k=4, gamma=None, beta=None, mean=FAKE, rstd=FAKE, act=0,
        go=ctypes.c_void_p(0x2000000), gdt=0, gx=OUT, gg=FAKE, gb=FAKE, ws=WS, wsb=1 << 28, st=None))
    for missing in ("x", "off", "mean", "rstd", "go", "gx"):
        assert call(**{missing: None}) == -1, missing
    assert call(gg=None) == -1 and call(gb=None) == -1 and "both or neither" in err(lib)
    assert call(gx=FAKE) == -1 and call(gx=ctypes.c_void_p(0x2000000)) == -1 and "overlap" in err(lib)
    assert call(ws=None) == -3 and call(wsb=8) == -3
    assert call(k=7) == -1 and call(gdt=2) == -1 and call(act=9) == -1 and call(f=4100, k=4) == -2


def test_group_norm_workspace(lib):
    n = ctypes.c_size_t(1)
    assert lib.tfg_group_norm_workspace_size(8, 4, 64, 8, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.tfg_group_norm_workspace_size(232965, 41, 128, 16, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.tfg_group_norm_workspace_size(100, 4, 64, 7, ctypes.byref(n)) == -1
    assert lib.tfg_group_norm_workspace_size(100, 4, 64, 8, None) == -1
    assert lib.tfg_group_norm_backward_workspace_size(100, 4, 64, 8, ctypes.byref(n)) == 0 and n.value >= 64 * 8
    assert lib.tfg_group_norm_backward_workspace_size(100, 4, 64, 7, ctypes.byref(n)) == -1


def tensors(ptrs, sizes, dtypes):
    return ((ctypes.c_void_p * len(ptrs))(*ptrs), (ctypes.c_int64 * len(sizes))(*sizes),
            (ctypes.c_int * len(dtypes))(*dtypes))


def test_clip_rejects(lib):
    base = [0x100000, 0x200000, 0x300000]

    def call(ptrs=base, sizes=(100, 7, 0), dtypes=(0, 1, 0), outs=(0x400000, 0x500000, None), clip=1.0, norm=FAKE, ws=WS,
             wsb=1 << 20, count=None):
        p, s, d = tensors(ptrs, sizes, dtypes)
        o = None if outs is None else (ctypes.c_void_p * len(outs))(*outs)
        return lib.tfg_clip_by_global_norm(len(ptrs) if count is None else count, p, s, d, clip, o, norm, ws, wsb, None)

    for clip in (0.0, -1.0, math.inf, math.nan):
        assert call(clip=clip) == -1, clip
    assert call(count=-1) == -1 and call(count=(1 << 20) + 1) == -2
    assert call(sizes=(100, -7, 0)) == -1 and call(sizes=(100, 1 << 46, 0)) == -2
    assert call(dtypes=(0, 5, 0)) == -1
    assert call(ptrs=[0x100000, None, 0x300000]) == -1 and call(outs=(None, 0x500000, None)) == -1
    assert call(ptrs=[0x100002, 0x200000, 0x300000]) == -1 and call(outs=(0x400000, 0x500001, None)) == -1
    assert call(outs=None) == -1 and call(norm=None) == -1
    assert call(ws=None) == -3 and call(wsb=64) == -3 and call(ws=ctypes.c_void_p(0x80000008)) == -1
    # an output on another tensor's input, on another output, on its own input by a shift,
    # and a tensor listed twice in place
    for ptrs, outs in [(base, (0x200000, 0x500000, None)), (base, (0x400000, 0x400000 + 396, None)),
                       (base, (0x100004, 0x500000, None)), ([0x100000, 0x100000, 0], (0x100000, 0x100000, None))]:
        assert call(ptrs=ptrs, outs=outs) == -1 and "overlap" in err(lib), (ptrs, outs)


def test_norm_rejects(lib):
    p, s, d = tensors([0x100000], [10], [0])
    assert lib.tfg_global_norm(1, p, s, d, None, WS, 1 << 20, None) == -1
    assert lib.tfg_global_norm(1, None, s, d, FAKE, WS, 1 << 20, None) == -1
    assert lib.tfg_global_norm(1, p, None, d, FAKE, WS, 1 << 20, None) == -1
    assert lib.tfg_global_norm(1, p, s, None, FAKE, WS, 1 << 20, None) == -1
    assert lib.tfg_global_norm(1, p, s, d, FAKE, None, 0, None) == -3
    n = ctypes.c_size_t(0)
    assert lib.tfg_global_norm_workspace_size(1, ctypes.byref(n)) == 0 and n.value > 0
    few = n.value
    assert lib.tfg_global_norm_workspace_size(5000, ctypes.byref(n)) == 0 and n.value > few
    assert lib.tfg_global_norm_workspace_size(-1, ctypes.byref(n)) == -1


def test_binding_refuses_cpu_tensors_and_wrong_types():
    import torch
    from paper_2101_11552_gb300 import tfg
    ids, x = torch.zeros(3, dtype=torch.int64), torch.zeros(3, 4)
    with pytest.raises(ValueError):
        tfg.tfg_embedding_lookup(x, ids)
    with pytest.raises(ValueError):
        tfg.tfg_group_ids(ids, 5)
    with pytest.raises(ValueError):
        tfg.tfg_group_norm(x, ids, 2)
    with pytest.raises(ValueError):
        tfg.tfg_global_norm([x])
    with pytest.raises(ValueError):
        tfg.tfg_clip_by_global_norm([x], 1.0)
