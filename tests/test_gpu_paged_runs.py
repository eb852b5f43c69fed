"""Paged decode in runs of many pages on the GPU: scores of millions."""
import numpy as np
import pytest

import _paged as P
import _paged_runs as R
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np
from test_gpu_paged import FMT

pytestmark = pytest.mark.gpu


def _records(k, v, fmt):
    """Pool of pages k, v [pages, hkv, 64, d] (fp16)."""
    num, hkv, _, d = k.shape
    pool = np.zeros((num, hkv, P.record_bytes(d, fmt)), np.uint8)
    for i in range(num):
        for head in range(hkv):
            for part, x in ((0, k), (1, v)):
                P.write_record(pool[i, head], d, fmt, part, x[i, head])
    return pool


def _call(pool, table, lens, q, fmt, copies=1, weights=None, decay=1.0, s=None):
    """The step with every kv head and its queries `copies` times; outputs of one copy, the others being the same."""
    b, hq, d = q.shape
    cache = h.PagedCache(to_gpu(np.tile(pool, (1, copies, 1))), to_gpu(table), to_gpu(np.asarray(lens, np.int32)), d, fmt)
    w = None if weights is None else to_gpu(weights)
    sg = None if s is None else to_gpu(np.tile(s, (copies, 1)))
    o, lse = h.hifa4_paged_decode_fwd(cache, to_gpu(np.tile(q, (1, copies, 1))), sg, page_weights=w, decay=decay)
    o, lse = to_np(o).reshape(b, copies, hq, d), to_np(lse).reshape(copies, hq, b)
    assert all(np.array_equal(o[:, c], o[:, 0], equal_nan=True) for c in range(copies))
    assert all(np.array_equal(lse[c], lse[0], equal_nan=True) for c in range(copies))
    return o[:, 0], lse[0], None if w is None else to_np(w)


@pytest.mark.parametrize("fmt,d,batch", [("fp16", 64, 24), ("fp16", 128, 16), ("fp16", 256, 8), ("hif4", 128, 16), ("hif4", 256, 8)])
@pytest.mark.parametrize("size", [2 ** 24, 2 ** 25, 2 ** 26, 2 ** 27, 2 ** 29, 2 ** 30])
def test_scores_of_millions(fmt, d, batch, size):
    """Scores whose fp32 steps are 2 binades and more, so that a reference some binades beside one is no number:
    maxima that differ by a few such steps within a run.  A score has two parts, the first one exact.  FP16: the
    second one is a multiple of the sum's step, so the sum is exact; HIF4: the groups' sum is rounded once.  The
    scale rounds once more, so the weights are known: powers of two."""
    fm, copies, num, pages = FMT[fmt], 64, 40, 13
    rng = np.random.default_rng(size)
    scale = np.float32(1.4426950408889634 / np.sqrt(d))
    big = 57344.0                                                 # 7 * 2^13: a key value that HIF4 holds
    first = 2.0 ** np.ceil(np.log2(size / scale / big / 8))       # eight query values of one digit
    step = 2.0 ** np.round(np.log2(size * 2.0 ** -24 / scale))    # (two of these are a step of the score)
    if fm == P.FP16:
        step = max(step, 2.0 ** (np.floor(np.log2(2 * size / scale)) - 23))
    k = np.zeros((num, 1, 64, d), np.float16)
    k[:, 0, :, :8] = big
    k[:, 0, :, d - 1] = np.maximum(rng.integers(0, 16, num)[:, None] - rng.integers(0, 9, (num, 64)), 0)
    v = rng.standard_normal((num, 1, 64, d)).astype(np.float16)
    pool = _records(k, v, fm)
    table = rng.integers(0, num, (batch, pages)).astype(np.int32)
    lens = [64 * pages - int(x) for x in rng.integers(0, 64, batch)]
    q = np.zeros((batch, 1, d), np.float16)
    q[:, 0, :8], q[:, 0, d - 1] = first, step
    assert np.isfinite(q).all() and min(r[2] - r[1] for r in R.plan(lens, copies, copies, d, fm)) >= 6
    o, lse, w = _call(pool, table, lens, q, fm, copies, np.zeros(table.shape, np.float32))
    kv = R.pool_values(pool, d, fm)
    for b, n in enumerate(lens):
        kk = kv[0, table[b], 0].reshape(-1, d)[:n]
        vv = kv[1, table[b], 0].reshape(-1, d)[:n]
        assert (kk[:, :8] == big).all()
        x = ((8 * first * big + step * kk[:, d - 1]).astype(np.float32) * scale).astype(np.float64)
        assert size <= x.max() < 2.001 * size and x.max() - x.min() >= 6
        e = np.exp2(x - x.max())
        p = e / e.sum()
        few = (4 * n + 64) * 2.0 ** -24                           # every key's sum in both halves of p, and the joins
        bound = 2 * few * (p @ np.abs(vv)) + 2.0 ** -11 * np.abs(p @ vv) + 2.0 ** -25
        if fm == P.HIF4:
            bound += 2.0 ** -19 * sum(p[j:j + 64].max() * np.abs(vv[j:j + 64]).sum(0) for j in range(0, n, 64))
        assert (np.abs(o[b, 0] - p @ vv) <= bound).all(), b
        assert abs(lse[0, b] - (x.max() + np.log2(e.sum())) * np.log(2)) <= 2.0 ** -23 * size * 2
        per = copies * np.add.reduceat(p, np.arange(0, n, 64))
        assert (np.abs(w[b] - per) <= few * per + 2.0 ** -60).all(), b
