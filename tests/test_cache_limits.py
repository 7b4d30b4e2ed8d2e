"""Sizes of the key-value cache at the ends of their range: decided on the host, nothing is launched."""
import ctypes as C

import pytest

from test_cache_host import L, P, UNSUPPORTED, batch, cache, plan_bytes, ws_bytes


@pytest.mark.parametrize("pages,heads,fits", [((2**31 - 2) // 8, 8, True), ((2**31 - 2) // 8 + 1, 8, False), (2**31 - 2, 1, True), (2**31 - 1, 1, False),
                                              (1 << 61, 8, False), ((1 << 61) + 3, 8, False), (1 << 52, 4096, False), ((1 << 63) - 1, 4096, False)])
def test_pools_of_more_pages_than_32_bits_count(pages, heads, fits):
    # pages * heads may pass 64 bits, too
    c, b = cache(pages=pages, heads=heads), batch(q_heads=heads)
    assert (plan_bytes(c, b) > 0) == fits and (ws_bytes(c, b) > 0) == fits
    if not fits:
        rc, rb = C.byref(c), C.byref(b)
        assert L.dybit_cache_plan(rc, rb, P(64), P(64), P(64), 1 << 40, None) == UNSUPPORTED
        assert L.dybit_cache_write(rc, rb, P(64), P(64), 1 << 20, 128, P(64), 1 << 20, 128, 1, 2, None) == UNSUPPORTED
        assert L.dybit_cache_read(rc, rb, P(64), P(64), 1 << 20, 128, P(64), 1 << 20, 128, 1, None) == UNSUPPORTED
        assert L.dybit_cache_attention(rc, rb, P(64), P(64), 1, 1 << 20, 128, P(64), 1 << 20, 128, None, 0.1, 1, 0, P(1024), 1 << 40, None) == UNSUPPORTED
