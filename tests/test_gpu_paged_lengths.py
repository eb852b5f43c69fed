"""Paged append on the GPU: sequences whose length was cut back, values that are
not finite."""
import numpy as np
import pytest

import _paged as P
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np
from test_gpu_paged import FMT

pytestmark = pytest.mark.gpu


def _append(cache, lens, k, v):
    """The last len(k[b]) tokens of each sequence."""
    cache.seq_lens.copy_(to_gpu(np.asarray(lens, np.int32)))
    cu = to_gpu(np.cumsum([0] + [len(x) for x in k]).astype(np.int32))
    h.hifa4_paged_append(cache, to_gpu(np.concatenate(k)), to_gpu(np.concatenate(v)), cu_new=cu)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_append_after_a_length_was_cut(fmt, d):
    """Rejected tokens: a length cut within the last append's page, to whole pages, or to nothing, then other tokens;
    the cache is that of the tokens that count.  FP16 pages: into an earlier page too."""
    import torch
    fm, hkv = FMT[fmt], 2
    rng = np.random.default_rng(d)
    had, cut, more = [100, 130, 66, 65, 200, 90], [70, 129, 64, 0, 128, 89], [5, 3, 70, 10, 1, 60]
    if fmt == "fp16":
        had, cut, more = had + [66, 200], cut + [62, 3], more + [4, 100]
    batch = len(had)
    table = rng.permutation(4 * batch).reshape(batch, 4).astype(np.int32)
    draw = lambda n: [rng.standard_normal((x, hkv, d)).astype(np.float16) for x in n]
    k0, v0, k1, v1 = draw(had), draw(had), draw(more), draw(more)
    caches = []
    for pieces in (True, False):
        cache = h.PagedCache.empty(4 * batch, batch, 4, hkv, d, fm)
        cache.block_table.copy_(to_gpu(table))
        if pieces:
            _append(cache, had, k0, v0)
            _append(cache, [c + m for c, m in zip(cut, more)], k1, v1)
        else:
            whole = [[np.concatenate([x[:c], y]) for x, c, y in zip(a, cut, b)] for a, b in ((k0, k1), (v0, v1))]
            _append(cache, [c + m for c, m in zip(cut, more)], *whole)
        caches.append(cache)
    lens = [c + m for c, m in zip(cut, more)]
    cu = to_gpu(np.cumsum([0] + lens).astype(np.int32))
    for a, b in zip(*[h.hifa4_paged_gather(c, cu, sum(lens)) for c in caches]):
        assert torch.equal(a, b)
    if fm == P.HIF4:                  # whole groups of V, what lies behind the last token included
        a, b = (to_np(c.pool) for c in caches)
        half = P.record_bytes(d, fm) // 2
        for i, n in enumerate(lens):
            for page in table[i, :-(-n // 64)]:
                assert np.array_equal(a[page, :, half:], b[page, :, half:]), (i, page)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_that_are_not_finite_stay_in_their_record(fmt, d):
    """Infinities and NaN in a token's K or V of one head change that page's record of that head alone (FP16: those
    values alone); later appends to other pages, and the steps of other sequences and heads, do not see them."""
    import torch
    fm, hkv = FMT[fmt], 3
    rng = np.random.default_rng(d + 9)
    lens = [150, 70]
    table = np.array([[3, 0, 5, 1], [2, 6, 4, 7]], np.int32)
    k, v = ([rng.standard_normal((n + 60, hkv, d)).astype(np.float16) for n in lens] for _ in range(2))
    q = to_gpu(rng.standard_normal((2, 6, d)).astype(np.float16))
    pools, outs = [], []
    for spoiled in (False, True):
        kk, vv = [x.copy() for x in k], [x.copy() for x in v]
        if spoiled:
            kk[0][70, 1, 3], kk[0][71, 1, d - 1], vv[0][80, 1, 5], vv[0][81, 1, 6] = np.inf, np.nan, -np.inf, np.nan
        cache = h.PagedCache.empty(8, 2, 4, hkv, d, fm)
        cache.block_table.copy_(to_gpu(table))
        cache.pool.zero_()
        _append(cache, lens, [x[:n] for x, n in zip(kk, lens)], [x[:n] for x, n in zip(vv, lens)])
        _append(cache, [n + 60 for n in lens], [x[n:] for x, n in zip(kk, lens)], [x[n:] for x, n in zip(vv, lens)])
        pools.append(to_np(cache.pool))
        outs.append([to_np(x) for x in h.hifa4_paged_decode_fwd(cache, q)])
    other = np.ones((8, hkv), bool)
    other[table[0, 1], 1] = False                                 # tokens 70 to 81: the sequence's second page
    assert np.array_equal(pools[0][other], pools[1][other])
    if fm == P.FP16:
        a, b = pools[0][0, 1].view(np.float16), pools[1][0, 1].view(np.float16)
        assert (a.view(np.uint16) != b.view(np.uint16)).sum() == 4
    (o0, l0), (o1, l1) = outs
    rows = np.ones((2, 6), bool)
    rows[0, 2:4] = False                                          # the queries of that head
    assert np.isfinite(o0).all() and np.array_equal(o0[rows], o1[rows]) and np.array_equal(l0.T[rows], l1.T[rows])
