"""The gated recurrence's waits for other tiles when they run out.

A build whose waits end at the first look (TFG_WAIT_LOOKS=0): a tile that does not find what it needs reports
TFG_ERR_TIMEOUT and goes on with NaN in its place, publishes what it has, and the kernel ends as ever.
"""
import pytest
import torch

from paper_2101_11552_gb300 import build, tfg
from test_gpu_gated_recurrence import batch, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hasty():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    path = build.build_library(defines=("TFG_WAIT_LOOKS=0",), only="gated_recurrence",
                               lib_path=build.os.path.join(build.OBJ_DIR, "libtfg_hasty.so"))
    yield path
    tfg.use_library(build.LIB_PATH)


def run(path, z, x, off, g, kind="sigmoid"):
    """Both directions by the library at path, the backward from the default build's forward."""
    whole = tfg.tfg_gated_recurrence(z, x, off, kind)
    tfg.check_status(whole.status)
    tfg.use_library(path)
    try:
        r = tfg.tfg_gated_recurrence(z, x, off, kind)
        b = tfg.tfg_gated_recurrence_backward(z, x, off, whole.checkpoints, g, kind)
        torch.cuda.synchronize()
    finally:
        tfg.use_library(build.LIB_PATH)
    return whole, r, b


@pytest.mark.parametrize("kind", ["sigmoid", "exp"])
@pytest.mark.parametrize("f,dt", [(64, "bf16"), (32, "f32"), (33, "f32")])
def test_a_wait_that_runs_out_is_reported(hasty, f, dt, kind):
    n = 60_000                                               # 469 tiles in a chain of 15 windows
    z, x = batch(n, f, kind, dt, 1)
    off, g = torch.tensor([0, n], device="cuda"), normal(n, f, 2, dt)
    whole, r, b = run(hasty, z, x, off, g, kind)
    assert int(r.status) == tfg.TFG_ERR_TIMEOUT and int(b.status) == tfg.TFG_ERR_TIMEOUT
    with pytest.raises(tfg.TfgError):
        tfg.check_status(r.status)
    # the device is as usable as before, and the default build's calls are as they were
    again = tfg.tfg_gated_recurrence(z, x, off, kind)
    tfg.check_status(again.status)
    assert torch.equal(again.out, whole.out) and torch.equal(again.final, whole.final)


def test_tiles_that_wait_for_none_need_no_second_look(hasty):
    """One tile, and sequences that end with their tiles: the same bits as the default build's."""
    for n, offsets in ((100, [0, 40, 100]), (1024, list(range(0, 1025, 128)))):
        z, x = batch(n, 40, "sigmoid", "f32", 1)
        off, g = torch.tensor(offsets, device="cuda"), normal(n, 40, 2)
        whole, r, b = run(hasty, z, x, off, g)
        tfg.check_status(r.status)
        tfg.check_status(b.status)
        want = tfg.tfg_gated_recurrence_backward(z, x, off, whole.checkpoints, g)
        assert torch.equal(r.out, whole.out) and torch.equal(b.gate, want.gate) and torch.equal(b.x, want.x)
