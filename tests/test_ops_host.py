"""What the worker's operators refuse and ask for on the host (CPU)."""
import ctypes as C
import os
import re

from paper_1805_08469_amd import gem as G

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gem.h")


def test_tokens_are_refused_where_their_positions_would_leave_32_bits():
    """A walk takes steps of 8 tokens and looks at the next one's end before it stops."""
    L, n = G.lib(), C.c_int64()
    most = int(re.search(r"#define GEM_TOKENS_MAX (\d+)", open(HEADER).read()).group(1))
    assert most == G.GEM_TOKENS_MAX and most + 3 * 8 <= 2**31 - 1
    for bad in (most + 1, 2**31 - 16, 2**31 - 8, 2**31 - 1):
        assert L.gem_scan_scratch(bad, 1, C.byref(n)) == G.GEM_EINVAL
        assert L.gem_scan_state_rows(bad, C.byref(n)) == G.GEM_EINVAL
    assert L.gem_scan_scratch(most, 1, C.byref(n)) == G.GEM_OK
    assert L.gem_scan_state_rows(most, C.byref(n)) == G.GEM_OK and n.value == most // 8
