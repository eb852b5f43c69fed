"""Paged decode in runs of many pages on the GPU: a maximum that moves within a
run, the weight of every page, plans of more runs than the call aims at, and
bounds that know what each rounding of the step may cost."""
import numpy as np
import pytest

import _paged as P
import _paged_runs as R
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np
from test_gpu_paged import FMT, _check

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


def _compare(got, want):
    o, lse, w = got
    ro, rl, rw, bo, bl, bw = want
    for a, x, bound, what in ((o, ro, bo, "o"), (lse, rl, bl, "lse"), (w, rw, bw, "weights")):
        if a is not None:
            _check(_Host(a), x, bound, what)


class _Host:
    """An array where a tensor is expected."""
    def __init__(self, a):
        self.a = a

    def detach(self):
        return self

    cpu = detach

    def numpy(self):
        return self.a


def _leveled(rng, num, d, levels, fmt):
    """Pages whose scores lie at levels[page, j] for the queries of kind j: channel 16 j holds the level, the query's
    other values of it.  Four kv heads, four queries each."""
    k = rng.standard_normal((num, 4, 64, d)).astype(np.float16)
    for j in range(4):
        k[:, :, :, 16 * j] = (levels[:, j, None, None] + rng.uniform(-0.5, 0.5, (num, 4, 64))).astype(np.float16)
    v = rng.standard_normal((num, 4, 64, d)).astype(np.float16)
    return _records(k, v, fmt)


def _queries(rng, batch, d):
    """Whole multiples of 2^-8 up to 32: digits hold them."""
    q = np.rint(rng.standard_normal((batch, 16, d)) * 64) / 256
    for head in range(16):
        for j in range(4):
            q[:, head, 16 * j] = 32.0 if j == head % 4 else 0.0
    return q.astype(np.float16)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d,batch", [(64, 24), (128, 16), (256, 8)])
@pytest.mark.parametrize("kind", ["moving", "flat"])
def test_runs_of_many_pages(fmt, d, batch, kind):
    """Two runs of six or seven pages a sequence.  "moving": a row's largest score rises within a run by less and by
    more than the softmax's reference tolerates, and falls by more than a hundred binades, at other places for each
    of a wave's four queries; pages that are none at a run's start and inside it."""
    fm, copies, num, pages = FMT[fmt], 16, 14, 13
    rng = np.random.default_rng(d)
    # binades of a level: 32 / sqrt(d) log2(e) each
    unit = np.sqrt(d) / 32 * np.log(2)
    binades = np.array([-170, -60, -25, -12, -6, -3, 0, 3, 6, 12, 20, 40, 90, 170], float)
    levels = np.stack([rng.permutation(binades) for _ in range(4)], 1) * unit if kind == "moving" else np.zeros((num, 4))
    pool = _leveled(rng, num, d, levels, fm)
    lens = [64 * pages - int(x) for x in rng.integers(0, 64, batch)]
    table = np.stack([rng.permutation(num)[:pages] for _ in range(batch)]).astype(np.int32)
    half = -(-pages // 2)
    table[1, 0] = table[2, half] = table[3, 3] = table[4, half + 2] = table[5, 5] = table[5, 6] = -1
    table[6, 1] = num
    q = _queries(rng, batch, d)
    w = rng.uniform(0, 1, table.shape).astype(np.float32)
    w[::2] = 0.0                                                  # (light pages show)
    runs = R.plan(lens, 16 * copies, 4 * copies, d, fm)
    assert [r[2] - r[1] >= 6 * R.units_of(d, fm) for r in runs] == [True] * (2 * batch)
    kv = R.pool_values(pool, d, fm)
    if kind == "moving":                                          # the case is what it is meant to be
        rise, fall = np.zeros(3, int), 0
        for b, begin, end in runs:
            for head in range(4):
                top = -np.inf
                for j in range(begin // R.units_of(d, fm), end // R.units_of(d, fm)):
                    if not 0 <= table[b, j] < num:
                        continue
                    x = (kv[0, table[b, j], 0] @ q[b, head].astype(float)).max() / np.sqrt(d) / np.log(2)
                    if np.isfinite(top):
                        rise += [0 < x - top < 8, 8 < x - top < 16, x - top > 16]
                        fall += x < top - 100
                    top = max(top, x)
        assert rise.min() >= 5 and rise[2] > 30 and fall > 30, (rise, fall)
    got = _call(pool, table, lens, q, fm, copies, w, 0.5)
    _compare(got, R.decode(q, kv, table, lens, fm, weights=w, decay=0.5, copies=copies))


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("lens", ["short", "long", "mixed"])
def test_plans_of_many_sequences(fmt, lens):
    """64 heads of 256 channels aim at 16 runs: more sequences than that, and fewer of which some need several."""
    fm, d, copies, num = FMT[fmt], 256, 16, 9
    rng = np.random.default_rng(len(lens))
    n = {"short": rng.integers(1, 65, 70), "long": rng.integers(1, 600, 15), "mixed": rng.integers(0, 260, 40)}[lens]
    n = [int(x) for x in n]
    target = R.run_target(64, 64, d, fm)
    runs = R.plan(n, 64, 64, d, fm)
    assert target == 16 and (len(n) >= target or lens == "long")
    if lens != "long":
        assert len(runs) > target
    assert max(r[2] - r[1] for r in runs) > (1 if lens == "short" else 2) * R.units_of(d, fm) or lens == "short"
    k, v = rng.standard_normal((2, num, 4, 64, d)).astype(np.float16)
    pool = _records(k, v, fm)
    table = rng.integers(0, num, (len(n), -(-max(n) // 64) + 1)).astype(np.int32)
    q = (np.rint(rng.standard_normal((len(n), 4, d)) * 64) / 64).astype(np.float16)
    w = np.zeros(table.shape, np.float32)
    got = _call(pool, table, n, q, fm, copies, w)
    _compare(got, R.decode(q, R.pool_values(pool, d, fm), table, n, fm, weights=w, copies=copies))


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_p_keeps_its_bits(fmt, d):
    """Values that cancel: a row of few keys whose output is far below its parts shows p's rounding, which that of o
    hides elsewhere.  One fp16 value for p would be out of the bound."""
    fm = FMT[fmt]
    rng = np.random.default_rng(5)
    batch, lens = 40, [2] * 40
    # one channel decides the score; the two keys weigh nearly the same, their values are opposite
    k = np.zeros((batch, 1, 64, d), np.float16)
    k[:, 0, 0, 0], k[:, 0, 1, 0] = 1.0, -1.0
    v = np.zeros((batch, 1, 64, d), np.float16)
    v[:, 0, 0], v[:, 0, 1] = 1.0, -1.0
    pool = _records(k, v, fm)
    table = np.arange(batch, dtype=np.int32)[:, None].copy()
    q = np.zeros((batch, 1, d), np.float16)
    q[:, 0, 0] = rng.uniform(0.001, 0.01, batch)
    kv = R.pool_values(pool, d, fm)
    want = R.decode(q, kv, table, lens, fm)
    if fmt == "fp16":
        wrong = R.decode(q, kv, table, lens, fm, rounded_p=True)[0]
        assert (np.abs(wrong - want[0]) > want[3]).any((1, 2)).sum() > batch // 2
    _compare(_call(pool, table, lens, q, fm), want)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("smooth", [False, True])
def test_queries_with_outlier_channels(fmt, d, smooth):
    """Channels of 16 and 64 times the others, as the query has them where Smooth-QK took them out of the keys."""
    fm = FMT[fmt]
    rng = np.random.default_rng(d + 1)
    lens = [200, 64, 700, 1]
    pages = [-(-n // 64) for n in lens]
    table = np.full((4, max(pages)), -1, np.int32)
    order = rng.permutation(sum(pages))
    for b, n in enumerate(pages):
        table[b, :n] = order[sum(pages[:b]):sum(pages[:b]) + n]
    k, v = rng.standard_normal((2, sum(pages), 2, 64, d)).astype(np.float16)
    q = rng.standard_normal((4, 8, d)).astype(np.float32)
    s = None
    if smooth:
        s = rng.uniform(0.5, 2.0, (2, d)).astype(np.float32)
        s[:, 5::d // 2] *= 64.0
        s[:, 9::d // 4] *= 16.0
    else:
        q[:, ::2, 5::d // 2] *= 64.0
        q[:, 1::2, 9::d // 4] *= 16.0
    pool = _records(k, v, fm)
    q = q.astype(np.float16)
    w = np.zeros(table.shape, np.float32)
    _compare(_call(pool, table, lens, q, fm, weights=w, s=s),
             R.decode(q, R.pool_values(pool, d, fm), table, lens, fm, s, w))


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
