"""The gated recurrence's flag for rows outside all sequences, beside gates: what is refused on the host (no GPU needed)."""
import ctypes
import os
import re

import pytest

FAKE, OUT, OUT2, OFF, WS, SMALL, MORE = (ctypes.c_void_p(0x100000 * k) for k in (1, 64, 96, 128, 160, 192, 224))


@pytest.fixture(scope="module")
def lib():
    from paper_2101_11552_gb300 import build, tfg
    build.build_library()
    return tfg.lib()


def test_the_binding_has_the_headers_flag():
    from paper_2101_11552_gb300 import build, tfg
    with open(os.path.join(build.ROOT, "include", "tfg.h")) as f:
        header = f.read()
    assert int(re.search(r"#define TFG_GATE_ZERO_OUTSIDE (\d+)", header).group(1)) == tfg.GATE_ZERO_OUTSIDE
    assert all(code & tfg.GATE_ZERO_OUTSIDE == 0 for code in tfg.GATES.values())


@pytest.mark.parametrize("kind", [2, 256 + 2, 512, 512 + 256, -1, -256])
def test_other_gates_are_refused_with_it_and_without(lib, kind):
    n, f = 100, 8
    assert lib.tfg_gated_recurrence(FAKE, f, MORE, f, 0, OFF, n, 1, f, kind, None, OUT, 0, None, None, None, 0, SMALL, None) == -1
    assert "unknown gate" in lib.tfg_last_error().decode()
    assert lib.tfg_gated_recurrence_backward(FAKE, f, MORE, f, 0, OFF, n, 1, f, kind, None, WS, None, 0, None, OUT, f, OUT2, f, None,
                                             None, 0, SMALL, None) == -1
    assert "unknown gate" in lib.tfg_last_error().decode()


def test_the_flag_changes_no_other_check(lib):
    """With it as without: an output that overlaps an input, a workspace too small."""
    n, f = 300, 8
    for kind in (0, 1, 256, 257):
        assert lib.tfg_gated_recurrence(FAKE, f, MORE, f, 0, OFF, n, 1, f, kind, None, FAKE, 0, None, None, WS, 1 << 20, SMALL, None) == -1
        assert "overlaps" in lib.tfg_last_error().decode()
        assert lib.tfg_gated_recurrence(FAKE, f, MORE, f, 0, OFF, n, 1, f, kind, None, OUT, 0, None, None, WS, 16, SMALL, None) != 0
