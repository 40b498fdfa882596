"""Refusals of the routing calls that only sizes no memory could hold reach: before any launch, on the host."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def qnn():
    from paper_2106_09886_b200 import build
    build.build()
    from paper_2106_09886_b200 import qnn as q
    return q


@pytest.mark.parametrize("top", [1, 2, 16, 32])
@pytest.mark.parametrize("tokens", [1 << 30, (1 << 32) + 5, 1 << 59, 1 << 60, (1 << 62) + 3, (1 << 63) - 1])
def test_slots_beyond_64_bits(qnn, tokens, top):
    """tokens * top is refused where it would wrap around as well."""
    buf = (ctypes.c_char * 512)()
    p = ctypes.c_void_p((ctypes.addressof(buf) + 255) // 256 * 256)      # aligned, never read
    assert qnn.lib.qnn_route_workspace(tokens, 64, top) == 0
    assert qnn.lib.qnn_route(p, 0, tokens, 64, 64, top, 0, None, 1, 1, 1.0, None, p, p, None, None, None, None, 0, None) == qnn.E_RANGE
    assert qnn.lib.qnn_route(p, 0, tokens, 64, 64, top, 0, None, 1, 1, 1.0, None, p, p, p, p, p, p, 1 << 40, None) == qnn.E_RANGE
    assert qnn.lib.qnn_route_backward(p, p, 0, tokens, 64, 64, top, 0, p, 1.0, p, 64, None) == qnn.E_RANGE
