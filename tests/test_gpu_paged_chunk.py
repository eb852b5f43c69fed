"""The attention of new tokens over the paged cache on the GPU, against tests/_paged_chunk.py (float64)."""
import numpy as np
import pytest
import torch

import _paged as P
import _paged_chunk as C
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np

pytestmark = pytest.mark.gpu

FMT = {"hif4": P.HIF4, "fp16": P.FP16}


def _inputs(rng, lens, hkv, d, smooth):
    k = [rng.standard_normal((max(n, 0), hkv, d)).astype(np.float32) for n in lens]
    if smooth:
        for x in k:
            x[:, :, ::37] *= 16
    v = [rng.standard_normal((max(n, 0), hkv, d)).astype(np.float16) for n in lens]
    s = (rng.uniform(0.4, 4.0, (hkv, d))).astype(np.float32) if smooth else None
    return [x.astype(np.float16) for x in k], v, s


def _table(rng, lens, spare=3, extra=1):
    pages = [(max(n, 0) + 63) // 64 for n in lens]
    order = rng.permutation(sum(pages) + spare)
    table = np.full((len(lens), max(pages + [1]) + extra), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _check(got, want, bound, what):
    got = to_np(got).astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), f"{what}: infinite elsewhere"
    err = np.abs(got - np.where(fin, want, 0.0))[fin]
    bad = ~(err <= bound[fin])
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, worst {np.max(err[bad] / bound[fin][bad]):.2f} times"


def _run(q, pool, table, lens, cu, d, fmt, s=None, max_new=None, **kw):
    cache = h.PagedCache(to_gpu(pool), to_gpu(table), to_gpu(np.asarray(lens, np.int32)), d, fmt)
    return h.hifa4_paged_chunk_fwd(cache, to_gpu(q), to_gpu(np.asarray(cu, np.int32)), None if s is None else to_gpu(s),
                                   max_new=max_new, **kw)


def _against(q, pool, table, lens, cu, d, fmt, s=None, max_new=None):
    o, lse = _run(q, pool, table, lens, cu, d, fmt, s, max_new)
    ro, rl, bo, bl, used = C.chunk(q, pool, table, lens, cu, fmt, s)
    _check(o[:len(used)][to_gpu(used)], ro[used], bo[used], "o")
    _check(lse[:, to_gpu(used)], rl[:, used], bl[:, used], "lse")
    return o, lse


def _case(seed, lens, new, hq, hkv, d, fmt, smooth=False, scale=1.0, holes=False, tight=True):
    rng = np.random.default_rng(seed)
    k, v, s = _inputs(rng, lens, hkv, d, smooth)
    table, num = _table(rng, lens)
    if holes:
        for b, n in enumerate(lens):
            if n > 128:
                table[b, 1] = (-1, num, 2 ** 31 - 1)[b % 3]
    pool = P.fill_pool(k, v, table, lens, num, fmt, s, junk=rng)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = (rng.standard_normal((int(cu[-1]), hq, d)) * scale).astype(np.float16)
    return _against(q, pool, table, lens, cu, d, fmt, s, max(list(new) + [1]) if tight else None)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([63, 64, 65], [63, 64, 65]), ([130, 0, 7], [5, 0, 7]), ([129, 64, 70], [2, 1, 66]),
                                      ([200], [137]), ([64, 128], [1, 64])])
def test_chunk_lengths(fmt, d, lens, new):
    _case(d + len(lens), lens, new, 4, 2, d, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 1), (13, 1), (17, 1), (40, 2), (33, 1), (64, 64)])
def test_chunk_heads(fmt, hq, hkv):
    _case(hq, [75, 37], [19, 3], hq, hkv, 64, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("grp", [1, 4, 7])
def test_chunk_smoothed(fmt, d, grp):
    _case(7, [150, 64, 99], [30, 1, 9], 2 * grp, 2, d, FMT[fmt], smooth=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_many_sequences(fmt):
    """More sequences than a wave has lanes; single tokens, chunks and empty rows mixed."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 140, 150)]
    new = [min(n, 1 if b % 8 else int(rng.integers(0, 60))) for b, n in enumerate(lens)]
    _case(1, lens, new, 2, 1, 64, FMT[fmt])
    _case(2, lens, new, 2, 1, 64, FMT[fmt], tight=False)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d,new", [(64, [3, 20, 1]), (128, [1, 1, 40]), (256, [2, 5, 9])])
def test_chunk_long(fmt, d, new):
    """Pages cut into runs that are joined."""
    _case(4, [9000, 20, 4097], [min(a, b) for a, b in zip(new, [9000, 20, 4097])], 4, 1, d, FMT[fmt], smooth=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[70, 40, 300, 129, 5], [1, 2, 3, 200, 1]])
def test_chunk_of_many_tiles(fmt, d, new):
    _case(8, [100, 40, 300, 257, 1400], new, 2, 2, d, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 9, 130, 3, 5], [140, 200, 260, 64, 400]])
def test_chunk_holes(fmt, d, new):
    """Pages that are none; rows that only see such; more new tokens than cached ones."""
    lens = [140, 200, 250, 64, 330]
    _case(17, lens, new, 4, 2, d, FMT[fmt], holes=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_peaked(fmt):
    """Large scores: the softmax rests on few keys, its maximum moves from page to page by hundreds."""
    _case(5, [500, 300], [6, 40], 8, 2, 128, FMT[fmt], scale=60.0)
    _case(6, [500, 300], [6, 40], 8, 2, 128, FMT[fmt], scale=1e-6)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("power", [24, 26, 27, 28, 30])
def test_chunk_huge_scores(fmt, power):
    """Scores of up to 2^30 (log2 units), whose neighbours in fp32 lie further apart than p's range: every row's keys
    are equal but for one twice as large, whose value the row takes exactly."""
    n, d = 200, 128
    k = np.full((n, 1, d), 2.0 ** 7, np.float16)
    q = np.full((20, 4, d), 2.0 ** (power - 7) / 128 * 8 * 2 ** 0.5 * np.log(2), np.float64)
    q = np.minimum(q, 60000.0).astype(np.float16)
    k *= np.float16(2.0 ** max(0, power - 26))
    k[50] *= 2
    v = np.random.default_rng(power).standard_normal((n, 1, d)).astype(np.float16)
    table = np.arange(4, dtype=np.int32)[None]
    pool = P.fill_pool([k], [v], table, [n], 4, FMT[fmt])
    o, lse = _run(q, pool, table, [n], [0, 20], d, FMT[fmt])
    _, vv, _ = P.cached(pool, table[0], n, 1, d, FMT[fmt])
    assert np.array_equal(to_np(o).astype(np.float64), np.broadcast_to(vv[50].astype(np.float16).astype(np.float64), (20, 4, d)))
    kk, _, _ = P.cached(pool, table[0], n, 1, d, FMT[fmt])
    want = (kk[50, 0] @ q.astype(np.float64).transpose(0, 2, 1)) / d ** 0.5
    assert np.allclose(to_np(lse).T.astype(np.float64), want, rtol=(d + 8) * 2.0 ** -24, atol=0)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_small_values(fmt):
    """Keys and values below fp16's normal range."""
    rng = np.random.default_rng(12)
    lens, new = [140], [9]
    k = [(rng.standard_normal((140, 1, 64)) * 2e-5).astype(np.float16)]
    v = [(rng.standard_normal((140, 1, 64)) * 4e-6).astype(np.float16)]
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, FMT[fmt])
    q = (rng.standard_normal((9, 2, 64)) * 1000).astype(np.float16)
    _against(q, pool, table, lens, np.array([0, 9]), 64, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_chunk_first_token_has_its_value(fmt, d):
    """A row that sees one key has that key's value, rounded to fp16, and the key's score."""
    rng = np.random.default_rng(d)
    k, v, _ = _inputs(rng, [70], 2, d, False)
    table, num = _table(rng, [70])
    pool = P.fill_pool(k, v, table, [70], num, FMT[fmt])
    q = rng.standard_normal((70, 6, d)).astype(np.float16)
    o, lse = _run(q, pool, table, [70], [0, 70], d, FMT[fmt])
    kk, vv, _ = P.cached(pool, table[0], 70, 2, d, FMT[fmt])
    for head in range(6):
        assert np.array_equal(to_np(o)[0, head], vv[0, head // 3].astype(np.float16))
        score = q[0, head].astype(np.float64) @ kk[0, head // 3] / d ** 0.5
        assert abs(float(lse[head, 0]) - score) <= 2.0 ** -18 + (d + 8) * 2.0 ** -24 * (np.abs(q[0, head]) @ np.abs(kk[0, head // 3])) / d ** 0.5


@pytest.mark.parametrize("new", [3, 40, 200])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bad", ["v", "k"])
def test_chunk_values_that_are_not_finite(bad, d, new):
    """An infinite or NaN value reaches the rows that see its token and no others, whatever lies in their tile."""
    rng = np.random.default_rng(new)
    lens = [260, 300]
    k, v, _ = _inputs(rng, lens, 2, d, False)
    x = v if bad == "v" else k
    x[0][259, 0, 3], x[0][258, 1, 7] = np.inf, np.nan
    x[0][260 - new, 0, 9] = -np.inf
    x[1][298, 0, 4], x[1][299, 0, 4] = np.inf, -np.inf
    x[1][max(0, 300 - new - 1), 1, 60] = np.nan
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, P.FP16, junk=rng)
    q = rng.standard_normal((2 * new, 4, d)).astype(np.float16)
    if bad == "k":
        q[:, :, [3, 4, 9]] = np.abs(q[:, :, [3, 4, 9]]) + np.float16(0.5)      # (an infinite score is positive or negative)
    cu = np.array([0, new, 2 * new], np.int32)
    o, lse = _run(q, pool, table, lens, cu, d, P.FP16, max_new=new)
    ro, rl, bo, bl, _ = C.chunk(q, pool, table, lens, cu, P.FP16)
    if bad == "k":          # a row whose largest score is infinite, or one of whose scores is NaN, is NaN as exp(inf - inf)
        poisoned = ~np.isfinite(rl.T) & ~(rl.T == -np.inf)
        assert poisoned.any() and np.isnan(to_np(o)[poisoned]).all() and np.isnan(to_np(lse).T[poisoned]).all()
        sound = ~poisoned
        _check(o[to_gpu(sound)], ro[sound], bo[sound], "o")
        _check(lse.t()[to_gpu(sound)], rl.T[sound], bl.T[sound], "lse")
    else:
        assert not np.isfinite(ro).all()
        _check(o, ro, np.where(np.isfinite(bo), bo, 0), "o")
        _check(lse, rl, bl, "lse")


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_rounds_smoothed_queries_once(fmt):
    """q s lies half way between fp16 numbers in fp32 but not exactly, or below their normal range.  A row that sees one
    key has its score as LSE: with one channel c of the key at 2^14 (on HIF4 pages what they hold for that: more than
    2^13, a few bits) that is q~_c k_c / 8, and another q~_c would be off by 2^-24 2^10 = 2^-14 and more, relatively by
    2^-11.  The score's product is exact; its scale, the reference, the
    exponent and the result are rounded, by less than 8 times 2^-24 of it, and log2 of the one p (2^7) by 2^-19."""
    rng = np.random.default_rng(40)
    d, heads, batch, at = 64, 64, 6, 5
    q = (rng.uniform(0.5, 2.0, (batch, heads, d)) * rng.choice([-1, 1], (batch, heads, d))).astype(np.float16)
    s = rng.uniform(0.5, 2.0, (heads, d)).astype(np.float32)
    half_way = rng.integers(1025, 2047, 32) / 1024 + 2.0 ** -11
    s[:32, at] = (half_way / np.abs(q[0, :32, at].astype(np.float64))).astype(np.float32)
    s[32:48, at] = (2.0 ** -16 * rng.uniform(0.5, 2.0, 16)).astype(np.float32)
    exact = q[:, :, at].astype(np.float64) * s[:, at].astype(np.float64)          # (35 bits)
    want = exact.astype(np.float16).astype(np.float64)
    twice = exact.astype(np.float32).astype(np.float16).astype(np.float64)
    assert (want != twice).sum() >= 4
    k = np.zeros((1, heads, d), np.float16)
    k[:, :, at] = 2.0 ** 14
    table = np.zeros((batch, 1), np.int32)
    pool = P.fill_pool([k], [np.ones_like(k)], table[:1], [1], 1, FMT[fmt])
    held = P.cached(pool, table[0], 1, heads, d, FMT[fmt])[0][0]
    assert np.array_equal(held != 0, k[0] != 0) and (held[:, at] > 2.0 ** 13).all()
    _, lse = _run(q, pool, table, [1] * batch, np.arange(batch + 1), d, FMT[fmt], s, 1)
    score = want * held[:, at] / 8
    assert (np.abs(to_np(lse).T - score) <= 2.0 ** -19 + 8 * 2.0 ** -24 * np.abs(score)).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [[16, 1], [17, 9], [32, 2], [33, 32]])
def test_chunk_rows_where_the_kinds_change(fmt, d, new):
    """16, 17, 32 and 33 rows of a sequence; the last page ends inside it."""
    _case(d + sum(new), [1300, 77], new, 2, 2, d, FMT[fmt], smooth=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("length", [1500, 9000])
def test_chunk_of_one_row_in_many_parts(fmt, d, length):
    """One token of one kv head: few rows in few parts and in many (joined by a wave, and by a workgroup's threads)."""
    _case(d, [length], [1], 8, 1, d, FMT[fmt], smooth=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 256])
def test_chunk_of_more_heads_than_workgroups(fmt, d):
    """As many kv heads as the chip holds workgroups, or more: one or two shares a head."""
    _case(d, [70, 130], [3, 40], 600, 600, d, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_cuts_sequences_behind_the_64th(fmt):
    """Long sequences among more than a wave has lanes: their tiles are cut, the plan walks on from one to the next."""
    rng = np.random.default_rng(41)
    lens = [int(x) for x in rng.integers(1, 30, 140)]
    for b in (0, 63, 64, 65, 127, 128, 139):
        lens[b] = 2000 + b
    new = [min(n, 3 if b % 2 else 50) for b, n in enumerate(lens)]
    _case(42, lens, new, 2, 1, 64, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_leaves_other_rows(fmt):
    """Rows behind the last sequence, and tokens beyond max_new, are left as they were."""
    rng = np.random.default_rng(20)
    lens, d = [200, 90, 64], 128
    k, v, s = _inputs(rng, lens, 2, d, True)
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, FMT[fmt], s, junk=rng)
    q = rng.standard_normal((60, 4, d)).astype(np.float16)
    cu = np.array([0, 33, 33, 40], np.int32)
    for max_new in (None, 33, 10, 1):
        o, lse = torch.full((60, 4, d), 7.0, dtype=torch.float16, device="cuda"), torch.full((4, 60), 7.0, device="cuda")
        got = _run(q, pool, table, lens, cu, d, FMT[fmt], s, max_new, out=o, lse=lse)
        assert got[0] is o and got[1] is lse
        ro, rl, bo, bl, used = C.chunk(q, pool, table, lens, cu, FMT[fmt], s)
        most = 60 if max_new is None else max_new
        for b in range(3):
            used[cu[b] + most:cu[b + 1]] = False
        _check(o[to_gpu(used)], ro[used], bo[used], "o")
        _check(lse[:, to_gpu(used)], rl[:, used], bl[:, used], "lse")
        assert (o[to_gpu(~used)] == 7.0).all() and (lse[:, to_gpu(~used)] == 7.0).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("cu", [[0, 40, 0, 40, 0, 40], [0, 0, 0, 0, 0, 0], [-5, 10, 10, 90, 3, 2 ** 31 - 1], [40, 30, 20, 10, 5, 0]])
def test_chunk_counts_outside_the_contract(fmt, cu):
    """Counts that are no prefix sums read and write no further than the buffers reach; what is written is right or
    nothing is."""
    rng = np.random.default_rng(21)
    lens, d = [200, 90, 64, 500, 1], 64
    k, v, _ = _inputs(rng, lens, 2, d, False)
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, FMT[fmt], junk=rng)
    q = rng.standard_normal((40, 4, d)).astype(np.float16)
    whole = torch.full((3, 40, 4, d), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((3, 4, 40), 7.0, device="cuda")
    for max_new in (40, 2):
        _run(q, pool, table, lens, cu, d, FMT[fmt], None, max_new, out=whole[1], lse=lse[1])
    assert (whole[0] == 7.0).all() and (whole[2] == 7.0).all() and (lse[0] == 7.0).all() and (lse[2] == 7.0).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_chunk_of_one_token_is_the_decode_step(fmt, d):
    """Both against the same float64 result, and against each other within the sum of both bounds."""
    rng = np.random.default_rng(22)
    lens = [700, 1, 64, 333]
    k, v, s = _inputs(rng, lens, 2, d, True)
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, FMT[fmt], s, junk=rng)
    q = rng.standard_normal((4, 8, d)).astype(np.float16)
    cache = h.PagedCache(to_gpu(pool), to_gpu(table), to_gpu(np.asarray(lens, np.int32)), d, FMT[fmt])
    od, ld = h.hifa4_paged_decode_fwd(cache, to_gpu(q), to_gpu(s))
    oc, lc = h.hifa4_paged_chunk_fwd(cache, to_gpu(q), torch.arange(5, dtype=torch.int32, device="cuda"), to_gpu(s), max_new=1)
    _, _, _, bo, bl, _ = P.decode(q, pool, table, lens, FMT[fmt], s)[:6]
    co, cl = C.chunk(q, pool, table, lens, np.arange(5), FMT[fmt], s)[2:4]
    assert (np.abs(to_np(od).astype(np.float64) - to_np(oc)) <= bo + co).all()
    assert (np.abs(to_np(ld).astype(np.float64) - to_np(lc)) <= bl + cl).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_beyond_4_gib(fmt):
    """Pages whose bytes begin behind 2^32, and the same bits from two calls."""
    rng = np.random.default_rng(23)
    d, hkv, lens = 128, 8, [400, 130]
    k, v, _ = _inputs(rng, lens, hkv, d, False)
    table, num = _table(rng, lens, spare=0)
    small = P.fill_pool(k, v, table, lens, num, FMT[fmt])
    bytes_ = small.shape[1] * small.shape[2]
    far = (2 ** 32 + 2 ** 30) // bytes_
    pool = torch.empty((far + num, hkv, small.shape[2]), dtype=torch.uint8, device="cuda")
    pool[far:] = to_gpu(small)
    q = rng.standard_normal((50, 8, d)).astype(np.float16)
    cu = np.array([0, 45, 50], np.int32)
    moved = np.where(table >= 0, table + far, -1).astype(np.int32)
    cache = h.PagedCache(pool, to_gpu(moved), to_gpu(np.asarray(lens, np.int32)), d, FMT[fmt])
    o, lse = h.hifa4_paged_chunk_fwd(cache, to_gpu(q), to_gpu(cu), max_new=45)
    o2, lse2 = _run(q, small, table, lens, cu, d, FMT[fmt], max_new=45)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_chunk_captured(fmt):
    """One graph, replayed with other lengths, counts, tables and queries: the bits of the eager call."""
    rng = np.random.default_rng(24)
    d, hq, hkv, batch, total, num = 128, 8, 2, 6, 90, 120
    pool = P.fill_pool(*_inputs(rng, [64 * num], hkv, d, False)[:2], np.arange(num, dtype=np.int32)[None], [64 * num], num, FMT[fmt])
    table = torch.full((batch, 40), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    cu = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    q = torch.zeros((total, hq, d), dtype=torch.float16, device="cuda")
    cache = h.PagedCache(to_gpu(pool), table, lens, d, FMT[fmt])
    o, lse = torch.zeros_like(q), torch.zeros((hq, total), device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.hifa4_paged_chunk_fwd(cache, q, cu, max_new=60, out=o, lse=lse)
    torch.cuda.synchronize()
    for step in range(5):
        n = [int(x) for x in rng.integers(0, 1200 if step else 60, batch)]
        new = [min(int(x), y) for x, y in zip(rng.integers(0, (1, 15)[step % 2] + 1, batch), n)]
        t, _ = _table(rng, n, spare=num - sum((x + 63) // 64 for x in n), extra=0)
        table.fill_(-1)
        table[:, :t.shape[1]] = to_gpu(t)
        lens.copy_(torch.tensor(n))
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape).astype(np.float16)))
        o.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eo, el = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
        h.hifa4_paged_chunk_fwd(cache, q, cu, max_new=60, out=eo, lse=el)
        assert torch.equal(o, eo) and torch.equal(lse, el)
        ro, rl, bo, bl, used = C.chunk(to_np(q), pool, to_np(table), n, to_np(cu), FMT[fmt])
        _check(o[to_gpu(used)], ro[used], bo[used], "o")
        _check(lse[:, to_gpu(used)], rl[:, used], bl[:, used], "lse")


def test_chunk_on_two_streams():
    """Calls of two streams at once, each with the workspace of its stream."""
    rng = np.random.default_rng(25)
    cases = []
    for i in range(2):
        lens, new = [3000 + 700 * i, 40], [9 + i, 4]
        k, v, _ = _inputs(rng, lens, 2, 128, False)
        table, num = _table(rng, lens)
        pool = P.fill_pool(k, v, table, lens, num, P.HIF4)
        q = rng.standard_normal((sum(new), 8, 128)).astype(np.float16)
        cache = h.PagedCache(to_gpu(pool), to_gpu(table), to_gpu(np.asarray(lens, np.int32)), 128, P.HIF4)
        cases.append((cache, to_gpu(q), to_gpu(np.array([0, new[0], sum(new)], np.int32))))
    alone = [h.hifa4_paged_chunk_fwd(*c, max_new=12) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(h.hifa4_paged_chunk_fwd(*cases[i], max_new=12))
    torch.cuda.synchronize()
    for (o, lse), many in zip(alone, got):
        for o2, lse2 in many:
            assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_chunk_binding_checks():
    cache = h.PagedCache.empty(4, 2, 2, 2, 64)
    q = torch.zeros((3, 4, 64), dtype=torch.float16, device="cuda")
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad in (dict(q=q[:, :, :32]), dict(q=q.float()), dict(cu=cu[:2]), dict(cu=cu.long()), dict(q=q[None]),
                dict(s=torch.zeros(2, 32, device="cuda")), dict(out=q[:2]), dict(lse=torch.zeros(4, 2, device="cuda")),
                dict(max_new=2 ** 31)):
        kw = dict(q=q, cu=cu)
        kw.update(bad)
        with pytest.raises(ValueError):
            h.hifa4_paged_chunk_fwd(cache, kw.pop("q"), kw.pop("cu"), kw.pop("s", None), **kw)
    with pytest.raises(h.Hifa4Error):
        h.hifa4_paged_chunk_fwd(cache, q[:, :3].contiguous(), cu)
    o, lse = h.hifa4_paged_chunk_fwd(cache, q[:0], cu)
    assert o.shape == (0, 4, 64) and lse.shape == (4, 0)


# --------------------------------------------------------------------------- the operators together
def _step(cache, rope, s, qkv, counts, free, num, shift, max_total, max_new, hq, hkv):
    """One step of a serving loop: pages, positions, rotation, append, attention."""
    cu, pos, slots = h.hifa4_paged_extend(cache.block_table, cache.seq_lens, counts, free, num, max_total, max_new=max_new, shift=shift)
    q, k = h.hifa4_rope(rope, pos, qkv[:, :hq], qkv[:, hq:hq + hkv])
    v = qkv[:, hq + hkv:].contiguous()
    h.hifa4_paged_append(cache, k, v, s, cu_new=cu, max_new=max_new)
    o, lse = h.hifa4_paged_chunk_fwd(cache, q, cu, s, max_new=max_new)
    return cu, pos, slots, q, k, v, o, lse


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_serving_loop(fmt, captured):
    """Prompts come in chunks, answers token by token, pages run short, sequences lose pages and end: every step's o
    against float64 over what the step before and the rotation have left, the pages' owners against a list."""
    rng = np.random.default_rng(30)
    batch, hq, hkv, d, num_pages, mp, max_total, max_new = 5, 4, 2, 64, 8, 12, 160, 100
    cache = h.PagedCache.empty(num_pages, batch, mp, hkv, d, FMT[fmt])
    rope = h.Rope(d, 32, scaling="parts", factor=4.0, original_len=64, low=1.0, high=8.0, magnitude=1.1)
    s = to_gpu(rng.uniform(0.5, 2.0, (hkv, d)).astype(np.float32))
    free = torch.arange(num_pages, dtype=torch.int32, device="cuda")
    num = torch.tensor([num_pages], dtype=torch.int32, device="cuda")
    shift = torch.zeros(batch, dtype=torch.int32, device="cuda")
    counts = torch.zeros(batch, dtype=torch.int32, device="cuda")
    qkv = torch.zeros((max_total, hq + 2 * hkv, d), dtype=torch.float16, device="cuda")
    graph = None
    if captured:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = _step(cache, rope, s, qkv, counts, free, num, shift, max_total, max_new, hq, hkv)
    refused = 0
    for step in range(14):
        ask = [0 if step % 5 == b else (int(rng.integers(40, 90)) if (step + b) % 4 == 0 else int(rng.integers(1, 4))) for b in range(batch)]
        ask = [min(a, 100) for a in ask]
        while sum(ask) > max_total:
            ask[int(np.argmax(ask))] //= 2
        before_lens, before_table = to_np(cache.seq_lens).copy(), to_np(cache.block_table).copy()
        counts.copy_(torch.tensor(ask, dtype=torch.int32))
        qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape).astype(np.float16)))
        want = C.extend(before_table, before_lens, ask, to_np(free), int(num), max_total, max_new, to_np(shift))
        if captured:
            graph.replay()
        else:
            out = _step(cache, rope, s, qkv, counts, free, num, shift, max_total, max_new, hq, hkv)
        torch.cuda.synchronize()
        cu, pos, slots, q, k, v, o, lse = out
        for x, y in zip((cache.block_table, cache.seq_lens, num, cu, pos, slots), want):
            assert np.array_equal(to_np(x).reshape(-1), np.asarray(y).reshape(-1))
        refused += int(np.diff(want[3]).sum() < sum(ask))
        # the new tokens are what the pages give back
        n = int(cu[-1])
        gk, gv = h.hifa4_paged_gather(cache, cu, max_total, max_tokens=max_new, starts=to_gpu(before_lens))
        if fmt == "fp16":
            assert torch.equal(gv[:n], v[:n])
            for b in range(batch):
                rows = slice(int(cu[b]), int(cu[b + 1]))
                assert torch.equal(gk[rows], torch.from_numpy((to_np(k)[rows].astype(np.float64) / to_np(s)).astype(np.float16)).cuda())
        lens = to_np(cache.seq_lens)
        ro, rl, bo, bl, used = C.chunk(to_np(q), to_np(cache.pool), to_np(cache.block_table), lens, to_np(cu), FMT[fmt], to_np(s))
        assert used.sum() == n
        _check(o[:n], ro[:n], bo[:n], "o")
        _check(lse[:, :n], rl[:, :n], bl[:, :n], "lse")
        if step % 3 == 2:       # two pages at most of each stay, the others go back; positions run on
            w = to_gpu(rng.random((batch, mp)).astype(np.float32))
            freed, gone = h.hifa4_paged_evict(cache.block_table, cache.seq_lens, w, budget=2, first=1, last=1)
            shift += 64 * gone
            h.hifa4_paged_release(freed, gone, free, num)
        if step % 4 == 3:       # a sequence ends
            b = step % batch
            to = torch.zeros(batch, dtype=torch.int32, device="cuda")
            to[b] = (int(cache.seq_lens[b]) + 63) // 64
            h.hifa4_paged_release(cache.block_table, to, free, num)
            cache.seq_lens[b] = 0
            shift[b] = 0
        lens = to_np(cache.seq_lens)
        owned = [int(x) for b in range(batch) for x in to_np(cache.block_table)[b, :(lens[b] + 63) // 64]]
        assert sorted(owned + [int(x) for x in to_np(free)[:int(num)]]) == list(range(num_pages))
        torch.zeros(1000, device="cuda").sum()
    assert refused
