"""The attention of new tokens over the paged cache at the ends of what its entry point accepts, on the GPU, against
tests/_paged_chunk.py (float64)."""
import numpy as np
import pytest
import torch

import _paged as P
import _paged_chunk as C
import paper_2607_04302_amd as h
from _gpu_util import to_gpu
from test_gpu_paged_chunk import FMT, _check, _inputs, _table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("new", [1, 5])
@pytest.mark.parametrize("hq", [1, 40])
def test_chunk_of_the_longest_table(fmt, new, hq):
    """2^25 - 1 places, six of them pages (the last one in use partly filled or full): what the rows see is what the
    same pages hold in a table of six places.  40 query heads of one kv head are many rows."""
    rng = np.random.default_rng(12)
    d, mp = 64, (1 << 25) - 1
    places = [0, 63, 64, 1 << 20, mp - 2, mp - 1]
    for last in (1, 64):
        short = [64 * 5 + last]
        k, v, s = _inputs(rng, short, 1, d, False)
        table, num = _table(rng, short, extra=0)
        pool = P.fill_pool(k, v, table, short, num, FMT[fmt], s, junk=rng)
        q = rng.standard_normal((new, hq, d)).astype(np.float16)
        ro, rl, bo, bl, _ = C.chunk(q, pool, table, short, [0, new], FMT[fmt])
        long_table = torch.full((1, mp), -1, dtype=torch.int32, device="cuda")
        long_table[0, places] = to_gpu(table[0, :6])
        cache = h.PagedCache(to_gpu(pool), long_table, to_gpu(np.array([64 * (mp - 1) + last], np.int32)), d, FMT[fmt])
        o, lse = h.hifa4_paged_chunk_fwd(cache, to_gpu(q), to_gpu(np.array([0, new], np.int32)))
        _check(o, ro, bo, "o")
        _check(lse, rl, bl, "lse")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,length", [(1, 1), (5, 70), (40, 40), (200, 200), (3, 9000)])
def test_chunk_of_scores_that_are_all_minus_infinity(d, new, length):
    """Rows all of whose scores are -inf (FP16 pages) have no weight to share out: o = 0 and lse = -inf, as of rows that
    see nothing; a row's first finite score takes all of it.  The same pages by one token of the decode step."""
    rng = np.random.default_rng(14)
    k, v, _ = _inputs(rng, [length], 1, d, False)
    k[0][:, 0, 3] = -np.inf
    if new > 1:
        k[0][-1, 0, 3] = 0.25                    # (the last token sees itself, finite)
    table, num = _table(rng, [length])
    pool = P.fill_pool(k, v, table, [length], num, P.FP16, junk=rng)
    q = rng.standard_normal((new, 2, d)).astype(np.float16)
    q[:, :, 3] = 1.0
    cache = h.PagedCache(to_gpu(pool), to_gpu(table), to_gpu(np.array([length], np.int32)), d, P.FP16)
    o, lse = h.hifa4_paged_chunk_fwd(cache, to_gpu(q), to_gpu(np.array([0, new], np.int32)))
    some = new - 1 if new > 1 else new
    assert bool((o[:some] == 0).all()) and bool((lse[:, :some] == -float("inf")).all())
    if new > 1:
        assert torch.equal(o[-1], to_gpu(v[0][-1]).expand(2, d)) and bool(torch.isfinite(lse[:, -1]).all())
    else:
        o, lse = h.hifa4_paged_decode_fwd(cache, to_gpu(q))
        assert bool((o == 0).all()) and bool((lse == -float("inf")).all())
