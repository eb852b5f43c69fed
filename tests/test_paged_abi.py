"""The paged cache's entry points reject invalid arguments with status codes
before any GPU work, the binding with ValueError (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import _paged as P
import paper_2607_04302_amd as h
from oracle import hif4

FAKE = 1 << 12          # an aligned non-NULL address; never dereferenced (validation fails first)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(h.LIB_PATH):
        pytest.skip("libhifa4.so not built")
    return h.load_library()


def _cache(**kw):
    base = dict(batch=2, num_heads_kv=2, head_dim=128, operands=0, num_pages=8, max_pages=4, pool=FAKE, block_table=FAKE,
                seq_lens=FAKE, v_tail=FAKE)
    base.update(kw)
    return h.PagedCacheDesc(**base)


def _append(lib, c, total=2, most=1, cu=None, k=FAKE, v=FAKE, s=None):
    return lib.hifa4_paged_append(ctypes.byref(c), total, most, cu, k, v, s, None)


def _gather(lib, c, total=2, most=1, cu=FAKE, starts=None, k=FAKE, v=FAKE):
    return lib.hifa4_paged_gather(ctypes.byref(c), total, most, cu, starts, k, v, None)


def _decode(lib, c, hq=4, q=FAKE, s=None, o=FAKE, lse=FAKE, w=None, wo=None, decay=1.0, ws=FAKE, nbytes=1 << 40):
    return lib.hifa4_paged_decode_fwd(ctypes.byref(c), hq, q, s, o, lse, w, wo, decay, ws, nbytes, None)


def _evict(lib, batch=2, mp=4, budget=2, first=0, last=1, ptrs=None):
    p = ptrs or [FAKE] * 8
    return lib.hifa4_paged_evict(batch, mp, *p[:3], budget, first, last, *p[3:], None)


def test_page_bytes():
    assert h.hifa4_paged_page_bytes(8, 128) == 8 * 2 * 64 * 128 * 36 // 64
    assert h.hifa4_paged_page_bytes(3, 64, h.OPERANDS_FP16) == 3 * 2 * 64 * 64 * 2
    for bad in ((0, 128, 0), (8, 96, 0), (8, 128, 2)):
        with pytest.raises(h.Hifa4Error):
            h.hifa4_paged_page_bytes(*bad)


@pytest.mark.parametrize("call", [_append, _gather, _decode])
def test_cache_is_checked(lib, call):
    assert call(lib, _cache(head_dim=96)) == -2
    assert call(lib, _cache(num_heads_kv=0)) == -1
    assert call(lib, _cache(operands=2)) == -1
    assert call(lib, _cache(batch=0)) == -1
    assert call(lib, _cache(max_pages=0)) == -1
    assert call(lib, _cache(num_pages=0)) == -1
    assert call(lib, _cache(max_pages=1 << 25)) == -2
    assert call(lib, _cache(max_pages=1 << 24, batch=1 << 8)) == -2
    for name in ("pool", "block_table", "seq_lens"):
        assert call(lib, _cache(**{name: None})) == -1
    for name in ("pool", "v_tail"):
        assert call(lib, _cache(**{name: FAKE + 8})) == -1
        assert "aligned" in h.hifa4_last_error()
    assert call(lib, _cache(seq_lens=FAKE + 2)) == -1


def test_append_and_gather_are_checked(lib):
    assert _append(lib, _cache(), total=-1, cu=FAKE) == -1
    assert _append(lib, _cache(), most=-1, cu=FAKE) == -1
    assert _append(lib, _cache(), total=3) == -1
    assert "one new token per sequence" in h.hifa4_last_error()
    assert _append(lib, _cache(), k=None) == -1
    assert _append(lib, _cache(), v=FAKE + 4) == -1
    assert _append(lib, _cache(), s=FAKE + 4) == -1
    assert _append(lib, _cache(), cu=FAKE + 1) == -1
    assert _append(lib, _cache(v_tail=None)) == -1
    assert "v_tail" in h.hifa4_last_error()
    assert _append(lib, _cache(batch=1 << 15, num_heads_kv=1 << 10, max_pages=4), total=1 << 20, most=1 << 20, cu=FAKE) == -2
    assert _append(lib, _cache(), total=0, cu=FAKE) == 0 and _append(lib, _cache(), most=0, cu=FAKE) == 0
    assert _gather(lib, _cache(), total=-1) == -1
    assert _gather(lib, _cache(), most=-1) == -1
    assert _gather(lib, _cache(), cu=None) == -1
    assert _gather(lib, _cache(), k=None) == -1
    assert _gather(lib, _cache(), v=FAKE + 2) == -1
    assert _gather(lib, _cache(), starts=FAKE + 2) == -1
    assert _gather(lib, _cache(batch=1 << 15, num_heads_kv=1 << 10), total=1 << 20, most=1 << 20) == -2
    assert _gather(lib, _cache(), total=0) == 0 and _gather(lib, _cache(), most=0) == 0


def test_decode_is_checked(lib):
    assert _decode(lib, _cache(), hq=0) == -1
    assert _decode(lib, _cache(), hq=3) == -2
    assert _decode(lib, _cache(batch=1 << 12), hq=1 << 12) == -2
    assert _decode(lib, _cache(), q=None) == -1
    assert _decode(lib, _cache(), o=FAKE + 8) == -1
    assert _decode(lib, _cache(), s=FAKE + 8) == -1
    assert _decode(lib, _cache(), lse=FAKE + 2) == -1
    assert _decode(lib, _cache(), w=FAKE) == -1 and _decode(lib, _cache(), wo=FAKE) == -1
    assert _decode(lib, _cache(), w=FAKE, wo=FAKE + 2) == -1
    assert _decode(lib, _cache(), w=FAKE, wo=FAKE, decay=float("nan")) == -1
    assert _decode(lib, _cache(), ws=None) == -3 and _decode(lib, _cache(), nbytes=16) == -3
    need = lib.hifa4_paged_decode_workspace_bytes(ctypes.byref(_cache()), 4, 0)
    more = lib.hifa4_paged_decode_workspace_bytes(ctypes.byref(_cache()), 4, 1)
    assert 0 < need < more
    assert _decode(lib, _cache(), w=FAKE, wo=FAKE, nbytes=more - 1) == -3
    assert lib.hifa4_paged_decode_workspace_bytes(ctypes.byref(_cache()), 3, 0) == 0
    assert lib.hifa4_paged_decode_workspace_bytes(None, 4, 0) == 0


def test_evict_is_checked(lib):
    assert _evict(lib, batch=0) == -1 and _evict(lib, mp=0) == -1
    assert _evict(lib, mp=1 << 25) == -2
    assert _evict(lib, last=0) == -1 and _evict(lib, first=-1) == -1 and _evict(lib, first=2) == -1
    for i in range(8):
        p = [FAKE] * 8
        p[i] = None
        assert _evict(lib, ptrs=p) == -1
        p[i] = FAKE + 2
        assert _evict(lib, ptrs=p) == -1


def test_launches_that_are_too_large_are_refused(lib):
    """2^24 workgroups of 256 threads (2^22 of 1024) are more than one launch holds."""
    big = _cache(batch=1 << 15, num_heads_kv=1 << 4, max_pages=64)      # 2^19 heads: 32 pages each are too many
    for call in (_append, _gather):
        assert call(lib, big, total=1 << 20, most=31 * 64, cu=FAKE) == -2
        assert "too many pages for one launch" in h.hifa4_last_error()
        assert call(lib, _cache(batch=1 << 20, num_heads_kv=1 << 12), total=1 << 20, most=1, cu=FAKE) == -2
    wide = _cache(batch=1 << 8, max_pages=(1 << 22) - 1)                 # 2^26 groups of 16 pages
    assert _decode(lib, wide, w=FAKE, wo=FAKE) == -2
    assert "page weights" in h.hifa4_last_error()
    assert lib.hifa4_paged_decode_workspace_bytes(ctypes.byref(wide), 4, 1) == 0
    assert lib.hifa4_paged_decode_workspace_bytes(ctypes.byref(wide), 4, 0) > 0
    assert _decode(lib, wide, ws=None) == -3                             # (no weights: that many pages are fine)
    assert _evict(lib, batch=1 << 22, mp=4) == -2
    # pages that runs take in halves: half as many
    halves = dict(batch=1 << 8, max_pages=1 << 21, operands=h.OPERANDS_FP16)
    assert _decode(lib, _cache(head_dim=256, **halves)) == -2
    assert _decode(lib, _cache(head_dim=128, **halves), ws=None) == -3


def test_counts_beyond_32_bits_are_refused(lib):
    """A count is never cut to 32 bits (2^32 tokens at most would otherwise mean none)."""
    class Cache:
        batch, heads_kv, head_dim, max_pages, device, _ref = 2, 2, 64, 4, torch.device("cuda", 0), None

    class Gpu:                                                           # as a GPU tensor of the right kind
        is_cuda, dtype = True, torch.float16
        device = Cache.device

        def __init__(self, *shape, dtype=torch.float16):
            self.shape, self.dtype = torch.Size(shape), dtype

        def dim(self):
            return len(self.shape)

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

    x, cu = Gpu(5, 2, 64), Gpu(3, dtype=torch.int32)
    for most in (1 << 32, -(1 << 40), 1 << 31):
        with pytest.raises(ValueError, match="max_new must fit 32 bits"):
            h.hifa4_paged_append(Cache, x, x, cu_new=cu, max_new=most)
        with pytest.raises(ValueError, match="max_tokens must fit 32 bits"):
            h.hifa4_paged_gather(Cache, cu, 5, max_tokens=most, k=x, v=x)
    with pytest.raises(ValueError, match="total_tokens must fit 32 bits"):
        h.hifa4_paged_gather(Cache, cu, 1 << 31)
    with pytest.raises(ValueError, match="k is"):
        h.hifa4_paged_append(Cache, Gpu(), x)
    table, lens, w = Gpu(2, 4, dtype=torch.int32), Gpu(2, dtype=torch.int32), Gpu(2, 4, dtype=torch.float32)
    for kw in ({"budget": 1 << 32}, {"budget": 2, "first": 1 << 32}, {"budget": 2, "last": (1 << 32) + 1}):
        with pytest.raises(ValueError, match="must fit 32 bits"):
            h.hifa4_paged_evict(table, lens, w, **kw)


def test_the_binding_refuses_before_the_library(lib):
    t = torch.zeros
    with pytest.raises(ValueError, match="pool must be a GPU tensor"):
        h.PagedCache(t((4, 2, 9216), dtype=torch.uint8), t((2, 4), dtype=torch.int32), t(2, dtype=torch.int32), 128)
    with pytest.raises(ValueError, match="GPU tensor"):
        h.hifa4_paged_evict(t((2, 4), dtype=torch.int32), t(2, dtype=torch.int32), t((2, 4)), 2)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_records_hold_every_value_once(d):
    """The layout that the tests read pages by: every (key, channel) has a place of its own, all places are used, and
    what is written is read back as the oracle's HIF4 values."""
    for part in (0, 1):
        code, nib, e2, e3, bit, base = P.hif4_places(d, part)
        half = P.record_bytes(d, P.HIF4) // 2
        assert len(set((2 * code + nib).ravel())) == 64 * d and code.min() == half * part
        assert len(set((8 * e2 + bit).ravel())) == 64 * d // 8 and len(set((8 * e3 + bit).ravel())) == 64 * d // 4
        assert len(set(base.ravel())) == d and base.max() == half * (part + 1) - 1
        assert not set(e2.ravel()) & set(e3.ravel()) and not set(base.ravel()) & set(code.ravel())
        x = np.random.default_rng(d).standard_normal((64, d)).astype(np.float16)
        rec = np.zeros(P.record_bytes(d, P.HIF4), np.uint8)
        P.write_record(rec, d, P.HIF4, part, x)
        got = P.read_record(rec, d, P.HIF4, part)
        want = hif4.quantize(x.reshape(64, -1, 64) if part == 0 else x.T)["xhat"]
        assert np.array_equal(got, want.reshape(64, d) if part == 0 else want.T)
        rec = np.zeros(P.record_bytes(d, P.FP16), np.uint8)
        P.write_record(rec, d, P.FP16, part, x)
        assert np.array_equal(P.read_record(rec, d, P.FP16, part), x)
    assert len(set(np.concatenate([P.fp16_places(d, 0).ravel(), P.fp16_places(d, 1).ravel()]))) == 128 * d
