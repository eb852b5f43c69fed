"""The paged cache in numpy: the records' layout, restated one value at a time
from its definition, and the operators over it in float64 (test data and
expected results only; the HIF4 codes are the oracle's)."""
import functools
import math

import numpy as np

from oracle import hif4, smooth

PAGE = 64
HIF4, FP16 = 0, 1


def record_bytes(d, fmt):
    return 72 * d if fmt == HIF4 else 256 * d


@functools.lru_cache(None)
def hif4_places(d, part):
    """(code byte, nibble, E2 byte, E3 byte, bit, base byte) of each (key, channel) of K (part 0) or V (part 1)."""
    g = d // 64
    out = np.zeros((6, 64, d), np.int64)
    for key in range(64):
        for ch in range(d):
            if part == 0:
                row, tile, elem = 16 * (key // 4 % 4) + 4 * (key // 16) + key % 4, ch // 64, ch % 64
            else:
                row, tile, elem = ch % 64, ch // 64, key
            t, n, w, i = row // 16, row % 16, elem // 8, elem % 8
            k, c = w // 2, w % 2
            lane = 16 * k + n
            o = 2304 * g * part
            code = o + 2048 * tile + 1024 * (t // 2) + 16 * lane + 8 * (t % 2) + 4 * c + i // 2
            if g == 1:
                e3 = i // 4
            else:
                e3 = 4 * (tile // 2) + 2 * (i // 4) + tile % 2
            out[:, key, ch] = (code, i % 2, o + 2176 * g + g * lane + tile, o + 2048 * g + 2 * g * lane + e3, 2 * t + c,
                               o + 2240 * g + 16 * g * (n // 4) + 16 * tile + 4 * t + n % 4)
    return out


@functools.lru_cache(None)
def fp16_places(d, part):
    """Index (in fp16 values) of each (key, channel)."""
    out = np.zeros((64, d), np.int64)
    for key in range(64):
        row = 16 * (key // 4 % 4) + 4 * (key // 16) + key % 4
        for ch in range(d):
            if part == 0:
                out[key, ch] = (((row // 16) * (d // 32) + ch // 32) * 64 + 16 * (ch // 8 % 4) + row % 16) * 8 + ch % 8
            else:
                out[key, ch] = 64 * d + ((ch // 16 * 2 + key // 8 % 2) * 64 + 16 * (key // 16) + ch % 16) * 8 + key % 8
    return out


def read_record(rec, d, fmt, part):
    """Values [64, d] (float64) of one record."""
    if fmt == FP16:
        return rec.view(np.float16)[fp16_places(d, part)].astype(np.float64)
    code, nib, e2, e3, bit, base = hif4_places(d, part)
    x = (rec[code] >> (4 * nib)) & 15
    sh = ((rec[e2] >> bit) & 1).astype(np.int64) + ((rec[e3] >> bit) & 1)
    return np.where(x & 8, -1.0, 1.0) * (x & 7) * hif4.E6M2_TABLE[rec[base].astype(np.int64)] / 4 * np.exp2(-sh.astype(float))


def write_record(rec, d, fmt, part, x):
    """Puts the values x [64, d] (fp16) into a record; HIF4 of whole groups."""
    if fmt == FP16:
        rec.view(np.float16)[fp16_places(d, part)] = x
        return
    code, nib, e2, e3, bit, base = hif4_places(d, part)
    groups = x.reshape(64, d // 64, 64) if part == 0 else x.T
    f = hif4.quantize(groups.astype(np.float64))

    def back(a, per):        # group fields -> [key, channel]
        a = np.repeat(a, per, -1)
        return a.reshape(64, d) if part == 0 else a.T

    n = back(f["u"] | (f["sign"].astype(np.uint8) << 3), 1)
    part_of = slice(2304 * (d // 64) * part, 2304 * (d // 64) * (part + 1))
    rec[part_of] = 0
    np.bitwise_or.at(rec, code.ravel(), (n << (4 * nib)).astype(np.uint8).ravel())
    np.bitwise_or.at(rec, e2.ravel(), (back(f["e2"], 8).astype(np.uint8) << bit.astype(np.uint8)).ravel())
    np.bitwise_or.at(rec, e3.ravel(), (back(f["e3"], 4).astype(np.uint8) << bit.astype(np.uint8)).ravel())
    rec[base.ravel()] = back(f["base"][..., None], 64).ravel()


def fill_pool(k, v, table, lens, num_pages, fmt, s=None, junk=None):
    """Pool [num_pages, hkv, bytes] holding the sequences k, v (lists of fp16 [L, hkv, d]).  Places behind a
    sequence's end and unused pages hold `junk` (a generator) or zeros; a V group is zero padded."""
    hkv, d = k[0].shape[1:]
    nb = record_bytes(d, fmt)
    pool = np.zeros((num_pages, hkv, nb), np.uint8)
    if junk is not None:
        pool = junk.integers(0, 256, pool.shape).astype(np.uint8)
    for b, n in enumerate(lens):
        kt = smooth.apply(k[b], k[b], s, hkv)[1] if s is not None else k[b]
        for j in range((n + PAGE - 1) // PAGE):
            page = table[b][j]
            if not 0 <= page < num_pages:
                continue
            m = min(PAGE, n - PAGE * j)
            for h in range(hkv):
                for part, x in ((0, kt), (1, v[b])):
                    y = np.zeros((PAGE, d), np.float16)
                    if fmt == FP16 and junk is not None:
                        y[:] = np.nan
                    y[:m] = x[PAGE * j:PAGE * j + m, h]
                    write_record(pool[page, h], d, fmt, part, y)
    return pool


def cached(pool, table_row, n, hkv, d, fmt):
    """(k, v float64 [n, hkv, d], present bool [n]) of a sequence."""
    k, v = np.zeros((2, n, hkv, d))
    there = np.zeros(n, bool)
    for j in range((n + PAGE - 1) // PAGE):
        page = table_row[j]
        m = min(PAGE, n - PAGE * j)
        if not 0 <= page < pool.shape[0]:
            continue
        there[PAGE * j:PAGE * j + m] = True
        for h in range(hkv):
            k[PAGE * j:PAGE * j + m, h] = read_record(pool[page, h], d, fmt, 0)[:m]
            v[PAGE * j:PAGE * j + m, h] = read_record(pool[page, h], d, fmt, 1)[:m]
    return k, v, there


def decode(q, pool, table, lens, fmt, s=None, weights=None, decay=1.0):
    """(o [B, Hq, D], lse [Hq, B], weights or None) in float64, and the bounds of a kernel that keeps scores and
    sums in fp32 and the weights p in 11 bits or more: |o| [B, Hq, D], lse [Hq, B], page weights [B, pages].

    Score error: D + 8 roundings of 2^-24 relative to sum |q k| / sqrt(D), in the worst order.  An error e of the
    scores moves p and the sums by e each way; p's own rounding is 2^-11 at most, o's 2^-11 of the result (and half
    a subnormal step); exponentials, partial sums and joins add 2^-18.

    On HIF4 pages a query value and a weight p are whole numbers of 32^-3 after scaling by a power of two that brings
    the largest of their 64 (a group of channels, a page's keys) to 8 or more, below or at 16.  Rounding to nearest
    moves one by half a step, 2^-16 of at least 8: by 2^-19 of that largest value.  So a score moves by 2^-19 of
    sum over the groups of max |q| sum |k| / sqrt(D) more, and o by 2^-19 of sum over the pages of max p sum |v|."""
    b_, hq, d = q.shape
    hkv = pool.shape[1]
    grp = hq // hkv
    o = np.zeros((b_, hq, d))
    lse = np.full((hq, b_), -np.inf)
    bo, bl = np.zeros((b_, hq, d)), np.zeros((hq, b_))
    w = None if weights is None else weights.astype(np.float64).copy()
    bw = None if weights is None else np.abs(w) * 2.0 ** -22
    for b, n in enumerate(lens):
        if w is not None:
            w[b, :(n + PAGE - 1) // PAGE] *= decay
        k, v, there = cached(pool, table[b], n, hkv, d, fmt)
        if not there.any():
            continue
        for h in range(hq):
            x = q[b, h].astype(np.float64)
            if s is not None:
                x = (x * s[h // grp].astype(np.float64)).astype(np.float16).astype(np.float64)
            kk, vv = k[there, h // grp], v[there, h // grp]
            sc = kk @ x / math.sqrt(d)
            m = sc.max()
            e = np.exp(sc - m)
            p = e / e.sum()
            o[b, h] = p @ vv
            lse[h, b] = m + math.log(e.sum())
            es = (d + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(x)).max() / math.sqrt(d)
            if fmt == HIF4:
                qm = np.repeat(np.abs(x).reshape(-1, 64).max(1), 64)
                es += 2.0 ** -19 * (np.abs(kk) @ qm).max() / math.sqrt(d)
                page = np.flatnonzero(there) // PAGE
                for j in set(page.tolist()):
                    bo[b, h] += 2.0 ** -19 * p[page == j].max() * np.abs(vv[page == j]).sum(0)
            bo[b, h] += (2.0 ** -11 + 2 * es + 2.0 ** -18) * (p @ np.abs(vv)) + 2.0 ** -11 * np.abs(o[b, h]) + 2.0 ** -25
            bl[h, b] = es + 2.0 ** -18 + 2.0 ** -22 * abs(lse[h, b])
            if w is not None:
                full = np.zeros(-(-n // PAGE) * PAGE)
                full[:n][there] = p
                per = full.reshape(-1, PAGE).sum(1)
                w[b, :len(per)] += per
                bw[b, :len(per)] += per * (2 * es + 2.0 ** -18) + 2.0 ** -30
    return o, lse, w, bo, bl, bw


def evict(table, lens, w, budget, first, last):
    out = [np.full_like(table, -1), np.array(lens, np.int32), np.zeros_like(w), np.full_like(table, -1),
           np.zeros(len(lens), np.int32)]
    mp = table.shape[1]
    for b in range(len(lens)):
        n = min(max(int(lens[b]), 0), PAGE * mp)
        pages = (n + PAGE - 1) // PAGE
        gone = []
        if pages > budget:
            key = [(-math.inf if math.isnan(x) else float(x)) for x in w[b]]
            order = sorted(range(first, pages - last), key=lambda j: (-key[j], math.isnan(w[b, j]), j))
            gone = sorted(order[budget - first - last:])
        keep = [j for j in range(pages) if j not in set(gone)]
        out[0][b, :len(keep)], out[2][b, :len(keep)] = table[b, keep], w[b, keep]
        out[3][b, :len(gone)], out[4][b] = table[b, gone], len(gone)
        out[1][b] = n - PAGE * len(gone)
    return out
