"""Refusals of the layer-norm, gated-recurrence and distillation entry points: every bad
argument is rejected on the host before anything is enqueued (no GPU needed)."""
import ctypes
import math

import pytest

FAKE = ctypes.c_void_p(0x100000)         # never dereferenced: every call below fails validation
OTHER = ctypes.c_void_p(0x900000)
THIRD = ctypes.c_void_p(0x2000000)
OUT = ctypes.c_void_p(0x40000000)
OUT2 = ctypes.c_void_p(0x50000000)
OUT3 = ctypes.c_void_p(0x60000000)
WS = ctypes.c_void_p(0x80000000)
SMALL = ctypes.c_void_p(0x700000)


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


def test_layer_norm_rejects(lib):
    call = caller(lib.tfg_layer_norm, dict(x=FAKE, xdt=0, res=OTHER, sdt=0, sum=THIRD, n=100, f=24, gamma=None, beta=None,
                                           eps=1e-5, out=OUT, odt=0, mean=None, rstd=None, st=None))
    assert call(n=-1) == -1 and call(f=0) == -1 and call(n=2**31) == -2 and call(f=(1 << 24) + 1) == -1
    assert call(n=2**31 - 1, f=1 << 24) == -2
    assert call(xdt=2) == -1 and call(odt=-1) == -1 and call(sdt=5) == -1
    for eps in (0.0, -1.0, math.inf, math.nan):
        assert call(eps=eps) == -1, eps
    for missing in ("x", "out"):
        assert call(**{missing: None}) == -1, missing
    assert call(sum=None) == -1 and call(res=None) == -1 and "both or neither" in err(lib)
    assert call(mean=SMALL) == -1 and call(rstd=SMALL) == -1
    assert call(out=FAKE) == -1 and call(out=OTHER) == -1 and call(out=THIRD) == -1 and "overlap" in err(lib)
    assert call(sum=FAKE) == -1 and call(sum=ctypes.c_void_p(0x900004)) == -1 and "overlap" in err(lib)
    assert call(gamma=OUT) == -1 and call(beta=THIRD) == -1
    for other in (FAKE, OTHER, THIRD, OUT, OUT2):           # statistics over an array, or over one another
        assert call(mean=other, rstd=OUT2) == -1 and call(mean=OUT2, rstd=other) == -1 and "overlap" in err(lib), other
    assert call(x=ctypes.c_void_p(0x100002)) == -1 and call(res=ctypes.c_void_p(0x900001), sdt=1) == -1 and "aligned" in err(lib)


def test_layer_norm_backward_rejects(lib):
    call = caller(lib.tfg_layer_norm_backward, dict(s=FAKE, sdt=0, n=100, f=24, gamma=None, mean=SMALL, rstd=SMALL, g=OTHER, gdt=0,
                                                    skip=THIRD, gs=OUT, xdt=0, gg=OUT2, gb=OUT3, ws=WS, wsb=1 << 30, st=None))
    for missing in ("s", "mean", "rstd", "g", "gs"):
        assert call(**{missing: None}) == -1, missing
    assert call(gg=None) == -1 and call(gb=None) == -1 and "both or neither" in err(lib)
    assert call(gs=FAKE) == -1 and call(gs=OTHER) == -1 and call(gs=ctypes.c_void_p(0x2000004)) == -1 and "overlap" in err(lib)
    assert call(gamma=OUT) == -1
    for other in (FAKE, OTHER, THIRD, OUT, SMALL):
        assert call(gg=other) == -1 and "overlap" in err(lib) and call(gb=other) == -1 and "overlap" in err(lib), other
    assert call(gg=OUT2, gb=OUT2) == -1 and "overlap" in err(lib)
    assert call(sdt=2) == -1 and call(gdt=2) == -1 and call(xdt=2) == -1
    assert call(ws=None) == -3 and call(wsb=8) == -3 and call(ws=ctypes.c_void_p(0x80000008)) == -1
    n = ctypes.c_size_t(0)
    assert lib.tfg_layer_norm_backward_workspace_size(100, 24, ctypes.byref(n)) == 0 and n.value >= 8 * 24
    assert lib.tfg_layer_norm_backward_workspace_size(100, 0, ctypes.byref(n)) == -1
    assert lib.tfg_layer_norm_backward_workspace_size(100, 24, None) == -1


SCAN = dict(gate=FAKE, gld=24, x=OTHER, xld=24, dt=0, off=SMALL, n=100, s=3, f=24, kind=0, init=None, out=OUT, odt=0, final=None,
            entering=None, ws=None, wsb=0, status=FAKE, st=None)


def test_recurrence_rejects(lib):
    call = caller(lib.tfg_gated_recurrence, SCAN)
    assert call(n=-1) == -1 and call(s=-1) == -1 and call(f=0) == -1
    assert call(n=2**31) == -2 and call(s=2**31 - 1) == -2
    assert call(n=2**31 - 1, f=4096, gld=4096, xld=4096) == -2           # more tiles than a grid holds
    assert call(gld=23) == -1 and call(xld=0) == -1 and "stride" in err(lib) and call(gld=1 << 45) == -2
    assert call(dt=2) == -1 and call(odt=3) == -1 and call(kind=2) == -1 and call(kind=-1) == -1
    for missing in ("gate", "x", "off", "out", "status"):
        assert call(**{missing: None}) == -1, missing
    for name in ("out", "final", "entering"):
        for other in (FAKE, OTHER, SMALL):
            assert call(**{name: other}) == -1, (name, other)
    assert call(init=THIRD, final=THIRD) == -1 and call(final=OUT) == -1 and call(entering=OUT) == -1 and "overlap" in err(lib)
    assert call(gate=ctypes.c_void_p(0x100002)) == -1
    assert call(n=129) == -3 and call(n=129, ws=WS, wsb=16) == -3 and "workspace" in err(lib)
    assert call(n=129, ws=ctypes.c_void_p(0x80000008), wsb=1 << 30) == -1


def test_recurrence_backward_rejects(lib):
    call = caller(lib.tfg_gated_recurrence_backward, dict(
        gate=FAKE, gld=24, x=OTHER, xld=24, dt=0, off=SMALL, n=100, s=3, f=24, kind=0, init=None, entering=THIRD, g=None, gdt=0,
        gfinal=None, gz=OUT, gzld=24, gx=OUT2, gxld=24, ginit=None, ws=None, wsb=0, status=FAKE, st=None))
    for missing in ("gate", "x", "off", "entering", "gz", "gx", "status"):
        assert call(**{missing: None}) == -1, missing
    assert call(gzld=23) == -1 and call(gxld=1) == -1
    for name in ("gz", "gx", "ginit"):
        for other in (FAKE, OTHER, SMALL, THIRD):
            assert call(**{name: other}) == -1, (name, other)
    assert call(gx=OUT) == -1 and call(ginit=OUT) == -1 and "overlap" in err(lib)
    # halves of one buffer share no value; a third of one and the half of another do
    half = ctypes.c_void_p(0x40000000 + 24 * 4)
    assert call(n=500, gzld=48, gxld=48, gx=half) == -3 and "workspace" in err(lib)
    assert call(gzld=48, gxld=48, gx=ctypes.c_void_p(0x40000000 + 20 * 4)) == -1 and "overlap" in err(lib)
    assert call(gzld=48, gxld=72, gx=half) == -1 and "overlap" in err(lib)
    assert call(n=500) == -3


def test_recurrence_workspace(lib):
    n = ctypes.c_size_t(1)
    ws = lib.tfg_gated_recurrence_workspace_size
    assert ws(128, 64, ctypes.byref(n)) == 0 and n.value == 0
    assert ws(129, 64, ctypes.byref(n)) == 0 and n.value >= 2 * 64 * 8
    assert ws(-1, 64, ctypes.byref(n)) == -1 and ws(5, 0, ctypes.byref(n)) == -1 and ws(5, 5, None) == -1


@pytest.mark.parametrize("suffix", ["", "32"])
def test_distillation_rejects(lib, suffix):
    d = dict(logits=FAKE, dt=0, n=10, v=50, ids=OTHER, teacher=THIRD, tdt=0, k=5, pad=-1, tau=1.0, w=None, loss=SMALL, stats=None,
             grad=OUT, status=FAKE, st=None)
    call = caller(getattr(lib, "tfg_distillation_loss" + suffix), d)
    assert call(n=-1) == -1 and call(v=0) == -1 and call(k=0) == -1
    assert call(n=2**31) == -2 and call(v=2**31 - 1) == -2 and call(k=1025) == -2
    assert call(dt=2) == -1 and call(tdt=2) == -1
    for tau in (0.0, -1.0, math.inf, math.nan, 1e-7, 1e7):
        assert call(tau=tau) == -1, tau
    for missing in ("logits", "ids", "teacher", "loss", "status"):
        assert call(**{missing: None}) == -1, missing
    for other in (FAKE, OTHER, THIRD):
        assert call(grad=other) == -1 and "overlap" in err(lib)
    for other in (FAKE, OTHER, THIRD, OUT):
        assert call(loss=other) == -1 and "overlap" in err(lib) and call(stats=other) == -1 and "overlap" in err(lib), other
    assert call(stats=SMALL) == -1 and call(w=SMALL) == -1 and "overlap" in err(lib)
    assert call(w=OUT) == -1 and call(stats=ctypes.c_void_p(0x700004)) == -1
    assert call(logits=ctypes.c_void_p(0x100002)) == -1 and call(grad=ctypes.c_void_p(0x40000002)) == -1
    for name in ("logits", "stats", "loss", "grad"):
        d.pop(name, None)
    back = caller(getattr(lib, "tfg_distillation_loss_backward" + suffix), dict(
        logits=FAKE, dt=0, n=10, v=50, ids=OTHER, teacher=THIRD, tdt=0, k=5, pad=-1, tau=1.0, w=None, stats=SMALL, gl=SMALL,
        grad=OUT, st=None))
    for missing in ("logits", "ids", "teacher", "stats", "gl", "grad"):
        assert back(**{missing: None}) == -1, missing
    for other in (FAKE, OTHER, THIRD, SMALL):
        assert back(grad=other) == -1 and "overlap" in err(lib)
    assert back(k=0) == -1 and back(tau=0.0) == -1


def test_binding_refuses_cpu_tensors_and_wrong_types():
    import torch
    from paper_2101_11552_gb300 import tfg
    x, off = torch.zeros(3, 4), torch.zeros(2, dtype=torch.int64)
    ids, top = torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2)
    for call in (lambda: tfg.tfg_layer_norm(x), lambda: tfg.tfg_layer_norm(None),
                 lambda: tfg.tfg_layer_norm_backward(x, None, x[:, 0], x[:, 0], x), lambda: tfg.tfg_gated_recurrence(x, x, off),
                 lambda: tfg.tfg_gated_recurrence(None, x, off), lambda: tfg.tfg_gated_recurrence_backward(x, x, off, x, x),
                 lambda: tfg.tfg_distillation_loss(x, ids, top),
                 lambda: tfg.tfg_distillation_loss_backward(x, ids, top, 1.0, top, x[:, 0])):
        with pytest.raises(ValueError):
            call()


def test_tile_rows_agree():
    import os
    import re
    from paper_2101_11552_gb300 import build, tfg
    text = open(os.path.join(build.ROOT, "include", "tfg.h")).read()
    assert tfg.RECURRENCE_TILE_ROWS == int(re.search(r"#define TFG_RECURRENCE_TILE_ROWS (\d+)", text).group(1))
