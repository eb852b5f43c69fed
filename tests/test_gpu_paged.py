"""The paged cache on the GPU: append, gather, decode and eviction against
tests/_paged.py (float64), their refusals of bad tables and lengths, and the
operators together in a serving loop, eager and captured."""
import numpy as np
import pytest

import _paged as P
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np

pytestmark = pytest.mark.gpu

FMT = {"hif4": P.HIF4, "fp16": P.FP16}


def _sequences(rng, lens, hkv, d, smooth):
    k = [rng.standard_normal((n, hkv, d)).astype(np.float32) for n in lens]
    if smooth:
        for x in k:
            x[:, :, ::37] *= 16
    v = [rng.standard_normal((n, hkv, d)).astype(np.float16) for n in lens]
    s = (rng.uniform(0.4, 4.0, (hkv, d))).astype(np.float32) if smooth else None
    return [x.astype(np.float16) for x in k], v, s


def _table(rng, lens, spare=3, extra=1):
    pages = [(n + 63) // 64 for n in lens]
    order = rng.permutation(sum(pages) + spare)
    mp = max(pages + [1]) + extra
    table = np.full((len(lens), mp), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _cache(pool, table, lens, d, fmt, tail=None):
    return h.PagedCache(to_gpu(pool), to_gpu(table), to_gpu(np.asarray(lens, np.int32)), d, fmt,
                        None if tail is None else to_gpu(tail))


def _check(got, want, bound, what):
    got = to_np(got).astype(np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fin), f"{what}: finite elsewhere"
    assert np.array_equal(got[~fin], want[~fin]), what
    err = np.abs(got - np.where(fin, want, 0.0))[fin]
    bad = err > bound[fin]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, worst {np.max(err[bad] / bound[fin][bad]):.2f} times"


# --------------------------------------------------------------------------- decode
def _decode_case(seed, lens, hq, hkv, d, fmt, smooth=False, weights=False, decay=0.75, scale=1.0, holes=False):
    rng = np.random.default_rng(seed)
    k, v, s = _sequences(rng, lens, hkv, d, smooth)
    table, num = _table(rng, lens)
    if holes:
        for b, n in enumerate(lens):
            if n > 128:
                table[b, 1] = (-1, num, 2 ** 31 - 1)[b % 3]
    pool = P.fill_pool(k, v, table, lens, num, fmt, s, junk=rng)
    q = (rng.standard_normal((len(lens), hq, d)) * scale).astype(np.float16)
    w = np.exp(rng.standard_normal(table.shape)).astype(np.float32) if weights else None
    cache = _cache(pool, table, lens, d, fmt)
    wt = None if w is None else to_gpu(w)
    o, lse = h.hifa4_paged_decode_fwd(cache, to_gpu(q), None if s is None else to_gpu(s), page_weights=wt, decay=decay)
    ro, rl, rw, bo, bl, bw = P.decode(q, pool, table, lens, fmt, s, w, decay)
    _check(o, ro, bo, "o")
    _check(lse, rl, bl, "lse")
    if weights:
        _check(wt, rw, bw, "weights")
    assert np.array_equal(to_np(cache.pool), pool)
    return o, lse


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens", [[1], [63, 64, 65], [0, 130, 0, 7], [700, 1, 64, 333, 0]])
def test_decode_lengths(fmt, d, lens):
    _decode_case(d + len(lens), lens, 4, 2, d, FMT[fmt], weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 1), (13, 1), (16, 1), (17, 1), (40, 2), (64, 64)])
def test_decode_heads(fmt, hq, hkv):
    _decode_case(hq, [150, 37], hq, hkv, 64, FMT[fmt], weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("grp", [1, 4, 7, 12])
def test_decode_smoothed(fmt, d, grp):
    _decode_case(7, [200, 64, 99], 2 * grp, 2, d, FMT[fmt], smooth=True, weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_decode_many_rows(fmt):
    """More sequences than a wave has lanes, and more than the runs that a call aims at."""
    rng = np.random.default_rng(3)
    _decode_case(1, [int(x) for x in rng.integers(0, 140, 150)], 2, 2, 64, FMT[fmt], weights=True)
    _decode_case(2, [int(x) for x in rng.integers(1, 70, 70)], 24, 12, 64, FMT[fmt])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_decode_few_keys_in_the_last_page(fmt, d):
    """Last pages of which a half, or all but a few of a lane's keys, are empty; pages that are none."""
    _decode_case(17, [8, 9, 72, 73, 136, 0, 56, 201], 4, 2, d, FMT[fmt], weights=True, holes=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_long(fmt, d):
    """Runs of one page and of many."""
    _decode_case(4, [9000, 20, 4097], 8, 2, d, FMT[fmt], smooth=True, weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_decode_peaked(fmt):
    """Large scores: the softmax rests on few keys, its maximum moves from page to page by hundreds."""
    _decode_case(5, [1000, 300], 8, 2, 128, FMT[fmt], scale=60.0, weights=True)
    _decode_case(6, [1000, 300], 8, 2, 128, FMT[fmt], scale=1e-6, weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("rising", [True, False])
def test_decode_small_weights_count(fmt, rising):
    """One key of weight 1 and thousands of weight 2^-18 or less, whose sum is what a coarse rounding of small
    weights loses; the heavy key first or last."""
    n, d = 4096, 64
    k = np.zeros((n, 1, d), np.float16)
    at = n - 1 if rising else 0
    k[:, 0, 0] = 1.0
    k[at, 0, 0] = 7.0
    q = np.zeros((1, 1, d), np.float16)
    q[0, 0, 0] = 18.5 * np.log(2) * 8 / 6
    v = np.ones((n, 1, d), np.float16)
    v[at] = -1.0
    table = np.arange(64, dtype=np.int32)[None].copy()
    pool = P.fill_pool([k], [v], table, [n], 64, FMT[fmt])
    cache = _cache(pool, table, [n], d, FMT[fmt])
    o, lse = h.hifa4_paged_decode_fwd(cache, to_gpu(q))
    ro, rl, _, bo, bl, _ = P.decode(q, pool, table, [n], FMT[fmt])
    _check(o, ro, bo, "o")
    _check(lse, rl, bl, "lse")


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_decode_not_finite(fmt, d):
    """A NaN or infinity in a query makes its own row NaN and no other; one in an FP16 page those of its head alone,
    and none behind the last token."""
    rng = np.random.default_rng(31)
    lens, hq, hkv = [150, 40, 9], 10, 2
    k, v, _ = _sequences(rng, lens, hkv, d, False)
    table, num = _table(rng, lens)
    pool = P.fill_pool(k, v, table, lens, num, FMT[fmt], junk=rng)
    q = rng.standard_normal((3, hq, d)).astype(np.float16)
    ro, rl, _, bo, bl, _ = P.decode(q, pool, table, lens, FMT[fmt])
    bad = np.zeros((3, hq), bool)
    for b, head, ch, x in ((0, 1, 3, np.nan), (1, 7, d - 1, np.inf), (2, 9, 0, -np.inf)):
        q[b, head, ch] = x
        bad[b, head] = True
    if fmt == "fp16":
        pool[table[0, 1], 1].view(np.float16)[P.fp16_places(d, 0)[5, 7]] = np.nan
        bad[0, hq // hkv:] = True
    o, lse = h.hifa4_paged_decode_fwd(_cache(pool, table, lens, d, FMT[fmt]), to_gpu(q))
    o, lse = to_np(o), to_np(lse)
    assert np.isnan(o[bad]).all() and np.isnan(lse.T[bad]).all()
    assert (np.abs(o[~bad] - ro[~bad]) <= bo[~bad]).all()
    assert (np.abs(lse.T[~bad] - rl.T[~bad]) <= bl.T[~bad]).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_decode_pages_that_are_none(fmt):
    _decode_case(8, [300, 200, 640, 100], 4, 2, 128, FMT[fmt], weights=True, holes=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_decode_is_deterministic_and_keeps_workspaces_apart(fmt):
    import torch
    rng = np.random.default_rng(9)
    lens = [2000, 77, 500]
    k, v, _ = _sequences(rng, lens, 2, 128, False)
    table, num = _table(rng, lens)
    cache = _cache(P.fill_pool(k, v, table, lens, num, FMT[fmt]), table, lens, 128, FMT[fmt])
    q = to_gpu(rng.standard_normal((3, 8, 128)).astype(np.float16))
    o, lse = h.hifa4_paged_decode_fwd(cache, q)
    ws = h.Workspace()
    need = h.hifa4_paged_decode_workspace_bytes(cache, 8)
    ws.get(need, q.device).fill_(255)                       # NaN everywhere
    for stream in (torch.cuda.Stream(), torch.cuda.Stream()):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            o2, lse2 = h.hifa4_paged_decode_fwd(cache, q)
        stream.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    o3, lse3 = h.hifa4_paged_decode_fwd(cache, q, workspace=ws)
    assert torch.equal(o, o3) and torch.equal(lse, lse3)
    out, l4 = torch.empty_like(o), torch.empty_like(lse)
    w, w2 = torch.ones(tuple(cache.block_table.shape), device="cuda"), torch.zeros(tuple(cache.block_table.shape), device="cuda")
    got = h.hifa4_paged_decode_fwd(cache, q, out=out, lse=l4, page_weights=w, weights_out=w2, decay=0.0)
    assert got[0] is out and got[1] is l4 and torch.equal(out, o) and torch.equal(l4, lse)
    assert bool((w == 1).all())
    used = torch.arange(w.shape[1], device="cuda") * 64 < cache.seq_lens[:, None]
    assert torch.equal(w2[~used], w[~used])
    assert torch.allclose(torch.where(used, w2, 0.0).sum(1), torch.full((3,), 8.0, device="cuda"), rtol=0, atol=1e-4)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d,hkv", [(64, 32), (128, 64), (256, 32)])
def test_decode_runs_longer_than_a_table_look_up(fmt, d, hkv):
    """Runs of more than 64 pages, on a table that names a few pages again and again: key j of page i counts as often
    as the table has i."""
    rng = np.random.default_rng(d)
    num, mp = 5, 6400 if d == 64 else 2200
    n = 64 * mp - 17
    k, v, _ = _sequences(rng, [64 * num], hkv, d, False)
    pool = P.fill_pool(k, v, np.arange(num)[None], [64 * num], num, FMT[fmt])
    table = rng.integers(0, num, (2, mp)).astype(np.int32)
    cache = _cache(pool, table, [n, 70], d, FMT[fmt])
    q = rng.standard_normal((2, hkv, d)).astype(np.float16)
    w = np.zeros((2, mp), np.float32)
    wt = to_gpu(w)
    o, lse = h.hifa4_paged_decode_fwd(cache, to_gpu(q), page_weights=wt)
    o, lse, wt = to_np(o).astype(np.float64), to_np(lse), to_np(wt)
    count = np.zeros((num, 64))
    for j in range(mp):
        count[table[0, j], :64 if j < mp - 1 else 47] += 1
    for head in range(hkv):
        kk, vv, _ = P.cached(pool[:, head:head + 1], np.arange(num), 64 * num, 1, d, FMT[fmt])
        s = kk[:, 0] @ q[0, head].astype(np.float64) / np.sqrt(d)
        e = np.exp(s - s.max()) * count.ravel()
        p = e / e.sum()
        assert abs(lse[head, 0] - (s.max() + np.log(e.sum()))) < 1e-4
        # p in 11 bits or more, the fp32 sums of 6400 pages (2^-24 a step at most), o to fp16
        bound = (2.0 ** -11 + 6400 * 2.0 ** -24) * (p @ np.abs(vv[:, 0])) + 2.0 ** -11 * np.abs(p @ vv[:, 0]) + 1e-6
        assert (np.abs(o[0, head] - p @ vv[:, 0]) <= bound).all()
    assert abs(wt[0].sum() - hkv) < 1e-2 and abs(wt[1, :2].sum() - hkv) < 1e-3 and (wt[1, 2:] == 0).all()


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_decode_batches_of_hundreds(fmt):
    """Batches over the 256 sequences that a wave keeps in registers, most of them empty, some with several runs."""
    rng = np.random.default_rng(12)
    lens = [int(x) for x in rng.integers(1, 90, 330) * (rng.random(330) < 0.3)]
    lens[5], lens[69], lens[261], lens[325], lens[329] = 1300, 900, 1500, 700, 0
    _decode_case(13, lens, 1, 1, 64, FMT[fmt], weights=True)


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_pages_beyond_four_gib(fmt):
    """A pool of more than 2^32 bytes: append, gather and decode at its end give what they give in a small pool."""
    import torch
    fm, hkv, d = FMT[fmt], 8, 128
    page = h.hifa4_paged_page_bytes(hkv, d, fm)
    big = (1 << 32) // page + 40
    rng = np.random.default_rng(6)
    lens = [500, 130]
    k, v, s = _sequences(rng, lens, hkv, d, True)
    table, num = _table(rng, lens)
    got = []
    for shift, pages in ((0, num), (big - num, big)):
        t = np.where(table >= 0, table + shift, -1).astype(np.int32)
        cache = h.PagedCache.empty(pages, 2, t.shape[1], hkv, d, fm)
        cache.block_table.copy_(to_gpu(t))
        cache.seq_lens.copy_(to_gpu(np.array(lens, np.int32)))
        cu = to_gpu(np.array([0, 500, 630], np.int32))
        h.hifa4_paged_append(cache, to_gpu(np.concatenate(k)), to_gpu(np.concatenate(v)), to_gpu(s), cu_new=cu)
        q = to_gpu(np.random.default_rng(1).standard_normal((2, 16, d)).astype(np.float16))
        got.append(h.hifa4_paged_gather(cache, cu, 630) + h.hifa4_paged_decode_fwd(cache, q, to_gpu(s)))
        torch.cuda.synchronize()
    assert cache.pool.numel() > 1 << 32
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    """Calls of two streams in flight together, each with a workspace of its own."""
    import torch
    rng = np.random.default_rng(21)
    lens = [5000, 2000, 64]
    k, v, _ = _sequences(rng, lens, 2, 128, False)
    table, num = _table(rng, lens)
    cache = _cache(P.fill_pool(k, v, table, lens, num, P.HIF4), table, lens, 128, P.HIF4)
    q = [to_gpu(rng.standard_normal((3, 8, 128)).astype(np.float16)) for _ in range(2)]
    want = [h.hifa4_paged_decode_fwd(cache, x) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(h.hifa4_paged_decode_fwd(cache, q[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])


def test_binding_refusals():
    import torch
    c = h.PagedCache.empty(4, 2, 3, 2, 64)
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")
    f32, i32 = torch.float32, torch.int32
    for args, kw in (((z(2, 4, 128),), {}), ((z(3, 4, 64),), {}), ((z(2, 4, 64, t=f32),), {}), ((z(2, 64, 4).transpose(1, 2),), {}),
                     ((z(2, 4, 64).cpu(),), {}), ((z(2, 4, 64), z(1, 64, t=f32)), {}), ((z(2, 4, 64),), {"out": z(2, 4, 128)}),
                     ((z(2, 4, 64),), {"lse": z(2, 4, t=f32)}), ((z(2, 4, 64),), {"weights_out": z(2, 3, t=f32)}),
                     ((z(2, 4, 64),), {"page_weights": z(2, 4, t=f32)}), ((z(4, 64),), {})):
        with pytest.raises(ValueError):
            h.hifa4_paged_decode_fwd(c, *args, **kw)
    with pytest.raises(h.Hifa4Error, match="multiple"):
        h.hifa4_paged_decode_fwd(c, z(2, 3, 64))
    for k, v, kw in ((z(2, 2, 64), z(2, 2, 128), {}), (z(2, 1, 64), z(2, 1, 64), {}),
                     (z(2, 2, 64), z(2, 2, 64), {"cu_new": z(2, t=i32)}), (z(2, 2, 64), z(2, 2, 64), {"s": z(2, 64)})):
        with pytest.raises(ValueError):
            h.hifa4_paged_append(c, k, v, **kw)
    with pytest.raises(h.Hifa4Error, match="one new token per sequence"):
        h.hifa4_paged_append(c, z(3, 2, 64), z(3, 2, 64))
    with pytest.raises(h.Hifa4Error, match="v_tail"):
        h.hifa4_paged_append(h.PagedCache(c.pool, c.block_table, c.seq_lens, 64), z(2, 2, 64), z(2, 2, 64))
    with pytest.raises(ValueError):
        h.hifa4_paged_gather(c, z(3, t=i32), 5, k=z(5, 2, 64), v=z(4, 2, 64))
    with pytest.raises(ValueError):
        h.hifa4_paged_gather(c, z(2, t=i32), 5)
    with pytest.raises(h.Hifa4Error, match="first"):
        h.hifa4_paged_evict(c.block_table, c.seq_lens, z(2, 3, t=f32), 2, 2, 1)
    for bad in ({"out_table": z(2, 4, t=i32)}, {"out_lens": z(3, t=i32)}, {"out_weights": z(2, 3)}, {"freed": z(2, 3, t=f32)},
                {"num_freed": z(2, 1, t=i32)}):
        with pytest.raises(ValueError):
            h.hifa4_paged_evict(c.block_table, c.seq_lens, z(2, 3, t=f32), 2, **bad)
    for args in ((c.pool[:, 0], c.block_table, c.seq_lens, 64), (c.pool, c.block_table[0], c.seq_lens, 64),
                 (c.pool, c.block_table, c.seq_lens[:1], 64), (c.pool, c.block_table, c.seq_lens, 128),
                 (c.pool, c.block_table, c.seq_lens, 64, h.OPERANDS_FP16), (c.pool, c.block_table, c.seq_lens, 64, 0, z(2, 64, 2, 128))):
        with pytest.raises(ValueError):
            h.PagedCache(*args)
    # nothing to do
    h.hifa4_paged_append(c, z(0, 2, 64), z(0, 2, 64), cu_new=z(3, t=i32))
    k, v = h.hifa4_paged_gather(c, z(3, t=i32), 0)
    assert k.shape == (0, 2, 64)
    o, lse = h.hifa4_paged_decode_fwd(c, z(2, 4, 64) + 1)
    assert bool((o == 0).all()) and bool((lse == float("-inf")).all())


# --------------------------------------------------------------------------- append and gather
@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("smooth", [False, True])
def test_append_in_pieces_equals_the_whole(fmt, d, smooth):
    """Prompts, single tokens and chunks that cross pages: after every append each page holds what writing the
    sequence at once gives, bit for bit, and a sequence that gets no token keeps its pages."""
    import torch
    hkv, fm = 3, FMT[fmt]
    rng = np.random.default_rng(d)
    steps = [[70, 1, 64, 0], [1, 1, 1, 1], [1, 62, 63, 0], [130, 0, 1, 63], [5, 3, 200, 1]]
    total = [sum(x[b] for x in steps) for b in range(4)]
    k, v, s = _sequences(rng, total, hkv, d, smooth)
    if fmt == "hif4":        # the quantizer's special cases
        from _edge import edge_rows
        edge_rows(k[0][:150], 1)
        edge_rows(v[2][64:200], 2)
        k[1][5], v[1][3] = 0, 0
    table, num = _table(rng, total)
    nb = P.record_bytes(d, fm)
    cache = h.PagedCache(to_gpu(rng.integers(0, 256, (num, hkv, nb)).astype(np.uint8)), to_gpu(table),
                         torch.zeros(4, dtype=torch.int32, device="cuda"), d, fm,
                         torch.full((4, 64, hkv, d), float("nan"), dtype=torch.float16, device="cuda") if fm == P.HIF4 else None)
    sg = None if s is None else to_gpu(s)
    have = np.zeros(4, int)
    for step in steps:
        new = np.array(step)
        kn = np.concatenate([k[b][have[b]:have[b] + new[b]] for b in range(4)])
        vn = np.concatenate([v[b][have[b]:have[b] + new[b]] for b in range(4)])
        have += new
        cache.seq_lens.copy_(to_gpu(have.astype(np.int32)))
        cu = None if step == [1, 1, 1, 1] else to_gpu(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        h.hifa4_paged_append(cache, to_gpu(kn), to_gpu(vn), sg, cu_new=cu, max_new=None if cu is None else int(new.max()))
        pool = to_np(cache.pool)
        want = P.fill_pool([x[:n] for x, n in zip(k, have)], [x[:n] for x, n in zip(v, have)], table, have, num, fm, s)
        for b, n in enumerate(have):
            gk, gv, _ = P.cached(pool, table[b], n, hkv, d, fm)
            wk, wv, _ = P.cached(want, table[b], n, hkv, d, fm)
            assert np.array_equal(gk, wk) and np.array_equal(gv, wv), (step, b)
            if fm == P.HIF4 and n:      # V's part of a page is its group, padding included
                for j in range((n + 63) // 64):
                    assert np.array_equal(pool[table[b, j], :, nb // 2:], want[table[b, j], :, nb // 2:]), (step, b, j)
    if fm == P.HIF4:
        tail = to_np(cache.v_tail)
        for b, n in enumerate(have):
            last = (n - 1) // 64 * 64
            assert np.array_equal(tail[b, :n - last], v[b][last:n])
            assert np.isnan(tail[b, max(n - last, min(n, 64)):]).all()
    # read back: everything, and pieces that begin and end inside pages
    for starts, counts in (([0] * 4, have), ([3, 64, 100, 0], [150, 3, 164, 65]), ([0, 60, 250, 65], [0, 9, 90, 5])):
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        out = [torch.full((int(cu[-1]) + 2, hkv, d), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
        gk, gv = h.hifa4_paged_gather(cache, to_gpu(cu), int(cu[-1]) + 2, max_tokens=int(max(counts)),
                                      starts=to_gpu(np.array(starts, np.int32)), k=out[0], v=out[1])
        assert gk is out[0] and gv is out[1]
        gk, gv = to_np(gk), to_np(gv)
        assert (gk[-2:] == 7).all() and (gv[-2:] == 7).all()
        for b in range(4):
            wk, wv, _ = P.cached(to_np(cache.pool), table[b], have[b], hkv, d, fm)
            wk, wv = (np.concatenate([x, np.zeros((400, hkv, d))])[starts[b]:starts[b] + counts[b]] for x in (wk, wv))
            assert np.array_equal(gk[cu[b]:cu[b + 1]], wk.astype(np.float16)), (starts, b)
            assert np.array_equal(gv[cu[b]:cu[b + 1]], wv.astype(np.float16)), (starts, b)


def test_append_writes_the_quantizers_codes():
    """The pages hold the codes of hifa4_quantize_qk and hifa4_quantize_v."""
    rng = np.random.default_rng(2)
    n, hkv, d = 200, 2, 128
    k, v, s = _sequences(rng, [n], hkv, d, True)
    cache = h.PagedCache.empty(4, 1, 4, hkv, d)
    cache.block_table.copy_(to_gpu(np.array([[2, 0, 3, 1]], np.int32)))
    cache.seq_lens.fill_(n)
    h.hifa4_paged_append(cache, to_gpu(k[0]), to_gpu(v[0]), to_gpu(s), cu_new=to_gpu(np.array([0, n], np.int32)))
    gk, gv, _ = P.cached(to_np(cache.pool), [2, 0, 3, 1], n, hkv, d, P.HIF4)
    from oracle import hif4
    _, _, kc, km = h.hifa4_quantize_qk(None, to_gpu(k[0][None]), to_gpu(s))
    vc, vm = h.hifa4_quantize_v(to_gpu(v[0][None]))
    wk = hif4.dequantize(hif4.unpack(to_np(kc), to_np(km).view(np.uint32)))            # [T, Hkv, G, 64]
    wv = hif4.dequantize(hif4.unpack(to_np(vc), to_np(vm).view(np.uint32)))[0]         # [NB, Hkv, D, 64]
    assert np.array_equal(gk, wk.reshape(n, hkv, d))
    assert np.array_equal(gv, wv.transpose(0, 3, 1, 2).reshape(-1, hkv, d)[:n])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_append_and_gather_stay_inside(fmt):
    """Tables with entries that are no pages, lengths and counts outside the contract: nothing but the sequences'
    own pages and rows is written."""
    import torch
    fm, hkv, d = FMT[fmt], 2, 64
    rng = np.random.default_rng(4)
    table = np.array([[0, -1, 5, 2], [7, 1 << 30, -5, 4], [1, 3, -1, -1], [6, -1, -1, -1]], np.int32)
    pool = rng.integers(0, 256, (7, hkv, P.record_bytes(d, fm))).astype(np.uint8)
    lens = np.array([1000, 200, -3, 30], np.int32)          # cut to 256 and 0
    cu = np.array([0, 160, 230, 300, 900], np.int32)        # past the input (400 rows), more than a sequence holds
    cache = _cache(pool, table, lens, d, fm, np.zeros((4, 64, hkv, d), np.float16) if fm == P.HIF4 else None)
    k = torch.randn(400, hkv, d, device="cuda").half()
    h.hifa4_paged_append(cache, k, k, cu_new=to_gpu(cu), max_new=100)
    after = to_np(cache.pool)
    # Sequence 0: 160 new ones at 96..255, the first 100 stored (96..195: pages -1, 5, 2); sequence 1: 70 at
    # 130..199 (its last two pages, none and 4); sequence 3: the last 30 of 100.
    for page in (0, 1, 3):
        assert np.array_equal(after[page], pool[page]), page
    assert len(cu) - 1 == len(lens)
    for b, first, stop, begin in ((0, 96, 196, 0), (1, 130, 200, 160), (3, 0, 30, 370)):
        gk, gv, there = P.cached(after, table[b], stop, hkv, d, fm)
        kn = to_np(k)[begin:begin + stop - first]
        at = np.arange(first, stop)[there[first:]]
        assert len(at)
        if fm == P.FP16:
            assert np.array_equal(gk[at], kn[at - first]) and np.array_equal(gv[at], kn[at - first])
        else:
            from oracle import hif4
            want = hif4.quantize(kn.astype(np.float64).reshape(-1, hkv, d // 64, 64))["xhat"].reshape(kn.shape)
            assert np.array_equal(gk[at], want[at - first])
    if fm == P.FP16:                                        # behind max_new: as it was (HIF4 clears what is unused)
        gk0 = P.cached(pool, table[0], 256, hkv, d, fm)[0]
        gk1 = P.cached(after, table[0], 256, hkv, d, fm)[0]
        assert np.array_equal(gk0[196:], gk1[196:], equal_nan=True)
    gk, gv = h.hifa4_paged_gather(cache, to_gpu(np.array([-5, 300, 300, 310, 10000], np.int32)), 320, max_tokens=310,
                                  starts=to_gpu(np.array([-7, 2 ** 31 - 1, 3, 40], np.int32)),
                                  k=torch.full((320, hkv, d), 7.0, device="cuda").half(),
                                  v=torch.full((320, hkv, d), 7.0, device="cuda").half())
    wk, wv, _ = P.cached(after, table[0], 256, hkv, d, fm)
    with np.errstate(over="ignore"):                      # (random bytes make values beyond fp16)
        wk, wv = wk.astype(np.float16), wv.astype(np.float16)
    for got, want in ((to_np(gk), wk), (to_np(gv), wv)):
        same = np.array_equal(got[:256], want, equal_nan=True)
        assert same and bool((got[256:] == 0).all())


# --------------------------------------------------------------------------- eviction
@pytest.mark.parametrize("mp,budget,first,last", [(1, 1, 0, 1), (9, 4, 1, 2), (9, 3, 1, 2), (40, 8, 0, 1), (513, 128, 1, 2),
                                                  (2500, 700, 4, 3), (2100, 2099, 0, 1), (70, 1, 0, 1)])
@pytest.mark.parametrize("kind", ["random", "ties", "special"])
def test_evict(mp, budget, first, last, kind):
    rng = np.random.default_rng(mp + budget)
    batch = 5
    lens = rng.integers(0, 64 * mp + 1, batch).astype(np.int32)
    lens[0], lens[1], lens[2] = 64 * mp, -5, 64 * mp + 1000
    table = rng.integers(-1, 10000, (batch, mp)).astype(np.int32)
    w = np.exp(rng.standard_normal((batch, mp)) * 3).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 3, (batch, mp)).astype(np.float32)
        w[0] = 1.0
    elif kind == "special":
        w[:, ::3] = np.nan
        w[:, 1::5] = np.inf
        w[:, 2::7] = -0.0
        w[:, 3::7] = 0.0
        w[:, 4::11] = -np.inf
        w[:, 5::13] = -1.0
        w[:, 6::17] = np.float32(1e-42)
    want = P.evict(table, lens, w, budget, first, last)
    args = [to_gpu(table), to_gpu(lens), to_gpu(w)]
    out = [a.clone() for a in args]
    freed, num = h.hifa4_paged_evict(*args, budget, first, last, out_table=out[0], out_lens=out[1], out_weights=out[2])
    for g, x, name in zip(out + [freed, num], want, ("table", "lens", "weights", "freed", "num_freed")):
        assert np.array_equal(to_np(g), x, equal_nan=name == "weights"), name
    assert np.array_equal(to_np(args[0]), table) and np.array_equal(to_np(args[2]), w, equal_nan=True)
    freed, num = h.hifa4_paged_evict(*args, budget, first, last)            # in place
    for g, x, name in zip(args + [freed, num], want, ("table", "lens", "weights", "freed", "num_freed")):
        assert np.array_equal(to_np(g), x, equal_nan=name == "weights"), "in place: " + name


# --------------------------------------------------------------------------- together
def _step(cache, state, s):
    """One step of a serving loop, on the device alone."""
    cache.seq_lens.add_(state["live"])
    h.hifa4_paged_append(cache, state["k"], state["v"], s)
    h.hifa4_paged_decode_fwd(cache, state["q"], s, page_weights=state["w"], decay=0.9, out=state["o"], lse=state["lse"])
    h.hifa4_paged_evict(cache.block_table, cache.seq_lens, state["w"], 4, 1, 1, freed=state["freed"], num_freed=state["num"])


@pytest.mark.parametrize("fmt", ["hif4", "fp16"])
def test_serving_loop_eager_and_captured(fmt):
    """Prompts, then steps of append, decode and eviction, against the same loop in float64; then the same steps
    from a captured graph, with eager work between the replays, bit for bit the eager loop."""
    import torch
    fm, hkv, hq, d, steps = FMT[fmt], 2, 6, 64, 70
    rng = np.random.default_rng(11)
    lens = np.array([250, 64, 0, 130, 400], np.int32)
    live = np.array([1, 1, 0, 1, 1], np.int32)
    k, v, s = _sequences(rng, list(lens + steps), hkv, d, True)
    q = rng.standard_normal((steps, 5, hq, d)).astype(np.float16)
    mp, num = 9, 48
    table = np.full((5, mp), -1, np.int32)
    order = rng.permutation(num)
    for b in range(5):
        table[b] = order[9 * b:9 * b + 9]        # pages for the whole run: an evicted sequence's table ends in -1

    def fresh():
        cache = h.PagedCache.empty(num, 5, mp, hkv, d, fm)
        cache.pool.fill_(0xFF)
        cache.block_table.copy_(to_gpu(table))
        cache.seq_lens.copy_(to_gpu(lens))
        sg = to_gpu(s)
        kn = to_gpu(np.concatenate([x[:n] for x, n in zip(k, lens)]))
        vn = to_gpu(np.concatenate([x[:n] for x, n in zip(v, lens)]))
        h.hifa4_paged_append(cache, kn, vn, sg, cu_new=to_gpu(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)),
                             max_new=int(lens.max()))
        z = torch.zeros
        state = {"live": to_gpu(live), "k": z((5, hkv, d), device="cuda").half(), "v": z((5, hkv, d), device="cuda").half(),
                 "q": z((5, hq, d), device="cuda").half(), "w": z((5, mp), device="cuda"),
                 "o": z((5, hq, d), device="cuda").half(), "lse": z((hq, 5), device="cuda"),
                 "freed": z((5, mp), dtype=torch.int32, device="cuda"), "num": z(5, dtype=torch.int32, device="cuda")}
        return cache, state, sg

    def inputs(state, i):
        state["k"].copy_(to_gpu(np.stack([k[b][lens[b] + i] for b in range(5)])))
        state["v"].copy_(to_gpu(np.stack([v[b][lens[b] + i] for b in range(5)])))
        state["q"].copy_(to_gpu(q[i]))

    def host_pages(cache):
        """The host's part: a page for every sequence whose next token opens one."""
        t, n = to_np(cache.block_table), to_np(cache.seq_lens)
        used = set(t[t >= 0].tolist())
        free = [p for p in range(num) if p not in used]
        for b in range(5):
            if live[b] and n[b] % 64 == 0 and t[b, n[b] // 64] < 0:
                t[b, n[b] // 64] = free.pop()
        cache.block_table.copy_(to_gpu(t))

    cache, state, sg = fresh()
    seen = []
    for i in range(steps):
        inputs(state, i)
        host_pages(cache)
        before = to_np(cache.block_table), to_np(state["w"])
        _step(cache, state, sg)
        n = to_np(cache.seq_lens) + 64 * to_np(state["num"])
        pool = to_np(cache.pool)
        ro, rl, rw, bo, bl, bw = P.decode(q[i], pool, before[0], n, fm, s, before[1], 0.9)
        _check(state["o"], ro, bo, f"o at step {i}")
        _check(state["lse"], rl, bl, f"lse at step {i}")
        seen.append([state[x].clone() for x in ("o", "lse", "w", "freed", "num")] + [cache.block_table.clone(), cache.seq_lens.clone()])
    assert sum(int(x[4].sum()) for x in seen) > 3

    cache, state, sg = fresh()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        inputs(state, 0)
        host_pages(cache)
        keep = [t.clone() for t in (cache.pool, cache.block_table, cache.seq_lens, state["w"])] + \
               [None if cache.v_tail is None else cache.v_tail.clone()]
        _step(cache, state, sg)                                 # warm: code objects are loaded
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            _step(cache, state, sg)
        for t, x in zip((cache.pool, cache.block_table, cache.seq_lens, state["w"], cache.v_tail), keep):
            if t is not None:
                t.copy_(x)
        for i in range(steps):
            inputs(state, i)
            host_pages(cache)
            graph.replay()
            torch.zeros(1 << 16, device="cuda").sum()           # the program's own work between replays
            stream.synchronize()
            got = [state[x] for x in ("o", "lse", "w", "freed", "num")] + [cache.block_table, cache.seq_lens]
            for a, x in zip(got, seen[i]):
                assert torch.equal(a, x), f"replay {i}"
