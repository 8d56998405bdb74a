"""Sizes whose index arithmetic would not fit 64 bits are refused by the host, and those beside them are not."""
import ctypes

import pytest

A = 1 << 20  # an address that is aligned and never read
NULL, LIMIT = -1, -6


def call(heads, kv, cap, n, cross, batch=1):
    import paper_2608_08081_b200 as iq
    from paper_2608_08081_b200 import binding as lib

    s, cb, k = lib._IqShape(batch, heads, kv, 128, cap, 2, 0.0), iq.iq_lloyd_max_codebook(128, 2).c(), lib._IqCache(A, A, A, A, None, 0, 0, 0)
    head = (ctypes.byref(s), A, ctypes.byref(cb), None, 0, heads * 128, 128, ctypes.byref(k), A, None, None, n)  # (no queries: refused behind the limits)
    return lib._lib.iq_cross_attention(*head, A, A, None, None, None) if cross else lib._lib.iq_chunk_attention(*head, 0, 0, A, A, None, None, None)


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("heads,kv,cap,n", [(1024, 1, 5 << 28, 1), (1024, 1, 5 << 28, 1000), (512, 1, (1 << 31) - (1 << 22), 1), (4096, 2, 1 << 30, 4)])
def test_a_tile_whose_share_of_blocks_does_not_fit(heads, kv, cap, n, cross):
    """Heads per KV head times rows times blocks: what chunk_blocks_before multiplies, in whole numbers."""
    assert (heads // kv) * (cap + n) * (cap // 128) >= 1 << 62
    assert call(heads, kv, cap, n, cross) == LIMIT


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("heads,kv,cap,n", [(64, 1, (1 << 31) - (1 << 22), 4096), (1024, 1, 1 << 28, 1024), (72, 1, 1 << 30, 1 << 16), (128, 8, 1 << 24, 1 << 20)])
def test_sizes_that_fit(heads, kv, cap, n, cross):
    group = heads // kv
    units = group * (cap + n + 1024) + 256
    tiles = kv * (-(-n * group // 256))
    assert units * (cap // 128 + 1) < 1 << 62 and units * tiles * 128 < 1 << 62
    assert call(heads, kv, cap, n, cross) == NULL
