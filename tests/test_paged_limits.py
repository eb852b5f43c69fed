"""What the paged cache's entry points refuse for its size, before any GPU work
(no GPU needed)."""
import ctypes

import pytest

import paper_2607_04302_amd as h
from test_paged_abi import FAKE, _append, _cache, _gather, lib  # noqa: F401


@pytest.mark.parametrize("operands", [h.OPERANDS_HIF4, h.OPERANDS_FP16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_appends_of_too_many_threads_are_refused(lib, d, operands):          # noqa: F811
    """A grid's threads are counted in 32 bits: 2^23 workgroups of 512 threads are too many, and 2^24 of any."""
    wide = d == 256 and operands == h.OPERANDS_HIF4
    kw = dict(head_dim=d, operands=operands, num_heads_kv=8, max_pages=64)
    # 1024 sequences of 8 heads: 2^23 workgroups with 1024 pages each, 2^24 with 2048
    for pages, refused in ((1024, wide), (2048, True)):
        tokens = 64 * (pages - 1) - 62                                       # (may begin in the middle of a page)
        c = _cache(batch=1024, **kw)
        if refused:
            assert _append(lib, c, total=1 << 20, most=tokens, cu=FAKE) == -2
            assert "too many pages for one launch (max_new of" in h.hifa4_last_error()
    assert _gather(lib, _cache(batch=1024, **kw), total=1 << 20, most=64 * 2047, cu=FAKE) == -2


def test_heads_and_sizes_beyond_32_bits_are_refused(lib):                     # noqa: F811
    """A count is never cut to 32 bits (2^32 + 8 heads are not 8)."""
    for args in (((1 << 32) + 8, 128), (8, (1 << 32) + 128), (8, 128, 1 << 32), (-(1 << 32) + 8, 128)):
        with pytest.raises(ValueError, match="must fit 32 bits"):
            h.hifa4_paged_page_bytes(*args)
    for kw in ({"heads_kv": (1 << 32) + 8}, {"head_dim": (1 << 32) + 128}, {"operands": 1 << 32}):
        with pytest.raises(ValueError, match="must fit 32 bits"):
            h.PagedCache.empty(**dict(dict(num_pages=1, batch=1, max_pages=1, heads_kv=8, head_dim=128), **kw))

    class Cache:
        _ref = ctypes.byref(_cache())
    with pytest.raises(ValueError, match="heads_q must fit 32 bits"):
        h.hifa4_paged_decode_workspace_bytes(Cache, (1 << 32) + 4)
    assert h.hifa4_paged_decode_workspace_bytes(Cache, 4) > 0
