"""What the worker's operators refuse and ask for on the host (CPU)."""
import ctypes as C
import os
import re

import pytest

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


@pytest.mark.parametrize("channels", [1, 64, 65, 128, 129, 512, 1001, 2048, 4096, 4100, 8192, 70000, 524288, 600000])
def test_scratch_never_falls_as_tokens_or_channels_grow(channels):
    """A handle made for the longest batch takes every shorter one."""
    before = 0
    for tokens in sorted({n + d for n in (0, 8, 16, 24, 32, 64, 128, 256, 1024, 4096, 16384, 32640, 32768, 65536, 131072,
                                          2**20, 2**24, G.GEM_TOKENS_MAX - 1) for d in (-1, 0, 1)} - {-1}):
        now = G.gem_scan_scratch(tokens, channels)
        assert now >= before, tokens
        assert G.gem_scan_scratch(tokens, channels + 1) >= now and G.gem_scan_scratch(tokens, max(1, channels // 2)) <= now
        before = now
    sizes = [G.gem_scan_scratch(t, channels) for t in range(0, 70000, 7)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("channels", [1, 64, 65, 130, 513, 1001, 2048, 4100, 8192, 70000, 600000])
def test_scratch_holds_every_shorter_batch(channels):
    """The bytes that a launch takes: 12 a channel of each run, whose length is halved from 128 to
    16 tokens until they leave 4096 rows of 128 channels."""
    def taken(tokens):
        length = 128
        while length > 16 and -(-tokens // length) * -(-channels // 128) < 4096:
            length //= 2
        runs = -(-tokens // length)
        return 0 if runs <= 1 else 12 * channels * runs

    worst = 0
    for tokens in range(0, 140000, 5):
        worst = max(worst, taken(tokens))
        assert G.gem_scan_scratch(tokens, channels) >= worst, tokens
