"""The attention of new tokens over the paged cache in float64, with the bounds of
the kernel's roundings; page tables dealt out and released one entry at a time."""
import math

import numpy as np

import _paged as P

PAGE = P.PAGE


def chunk(q, pool, table, lens, cu, fmt, s=None):
    """(o [T, Hq, D], lse [Hq, T], their bounds, rows that a sequence has [T]).

    Scores: the products of fp16 values are exact in fp32; D + 8 roundings of 2^-24
    (sums, scale, difference to the reference) relative to the largest sum |q k| /
    sqrt(D) that the row sees: es.  On HIF4 pages a value below 2^-14 is rounded by up
    to 2^-24: a score by 2^-24 sum |q| / sqrt(D), o by 2^-24.  An error e of the scores
    moves p and its sum by e each way.  p is rounded to fp16: by 2^-11 of itself, or by
    2^-25 where the heaviest key so far counts at least 2^7, 2^-32 of that one's; o =
    sum p^ v / sum p^ moves by sum |p^ - p| |v - o|.  fp32 sums: one rounding of 2^-24
    per 32 keys and 64 more; exponentials and joins 2^-18.  o is rounded by 2^-11 of
    itself, or 2^-25."""
    t_, hq, d = q.shape
    hkv = pool.shape[1]
    grp = hq // hkv
    o, lse = np.zeros((t_, hq, d)), np.full((hq, t_), -np.inf)
    bo, bl = np.zeros((t_, hq, d)), np.zeros((hq, t_))
    used = np.zeros(t_, bool)
    for b, n in enumerate(lens):
        n = int(min(max(n, 0), PAGE * table.shape[1]))
        k, v, there = P.cached(pool, table[b], n, hkv, d, fmt)
        m = cu[b + 1] - cu[b]
        for i in range(m):
            row, pos = cu[b] + i, n - m + i
            used[row] = True
            seen = np.flatnonzero(there[:max(0, pos + 1)])
            if not len(seen):
                continue
            for h in range(hq):
                x = q[row, h].astype(np.float64)
                if s is not None:
                    x = (x * s[h // grp].astype(np.float64)).astype(np.float16).astype(np.float64)
                kk, vv = k[seen, h // grp], v[seen, h // grp]
                with np.errstate(invalid="ignore"):
                    sc = kk @ x / math.sqrt(d)
                    top = sc.max()
                    e = np.exp(sc - top)
                    p = e / e.sum()
                    o[row, h] = p @ vv
                    lse[h, row] = top + math.log(e.sum())
                    es = (d + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(x)).max() / math.sqrt(d)
                    if fmt == P.HIF4:
                        es += 2.0 ** -24 * np.abs(x).sum() / math.sqrt(d)
                        bo[row, h] += 2.0 ** -24
                    sums = 2.0 ** -18 + (len(seen) / 32 + 64) * 2.0 ** -24
                    weighed, size = p @ np.abs(vv), np.abs(o[row, h])
                    bo[row, h] += 2.0 ** -11 * (weighed + size) + 2.0 ** -32 * p.max() * (np.abs(vv).sum(0) + len(seen) * size)
                    bo[row, h] += (2 * es + sums) * weighed + 2.0 ** -11 * size + 2.0 ** -25
                    bl[h, row] = es + sums + 2.0 ** -22 * abs(lse[h, row])
    return o, lse, bo, bl, used


def extend(table, lens, counts, free, num_free, max_total, max_new, shift=None):
    """(table, lens, number free, cu, positions, slots) after the pages were dealt out."""
    table, lens = table.copy(), np.array(lens, np.int64)
    most = PAGE * table.shape[1]
    top = int(min(max(num_free, 0), len(free)))
    stack = [int(x) for x in free[:top]]
    cu, positions, slots = [0], np.full(max_total, -1, np.int32), np.full(max_total, -1, np.int64)
    asked = needed = 0
    for b in range(len(lens)):
        have = int(min(max(lens[b], 0), most))
        n = max(0, int(counts[b]))
        if n > min(max_new, most - have):
            n = 0
        first, last = -(-have // PAGE), -(-(have + n) // PAGE)
        asked += n
        needed += last - first
        if asked > max_total or (last > first and needed > top):
            n = 0
        else:
            for j in range(first, last):
                table[b, j] = stack.pop()
        for i in range(n):
            page = int(table[b, (have + i) // PAGE])
            positions[cu[-1] + i] = have + i + (0 if shift is None else int(shift[b]))
            slots[cu[-1] + i] = page * PAGE + (have + i) % PAGE if page >= 0 else -1
        lens[b] = have + n
        cu.append(cu[-1] + n)
    return table, lens.astype(np.int32), len(stack), np.array(cu, np.int32), positions, slots


def release(table, to, free, num_free, first=None):
    """(stack, number free) after the entries were put back."""
    free = free.copy()
    pages = []
    for b in range(len(table)):
        lo = 0 if first is None else max(0, int(first[b]))
        pages += [int(x) for x in table[b, lo:max(lo, min(int(to[b]), table.shape[1]))] if x >= 0]
    n = int(min(max(num_free, 0), len(free)))
    for page in reversed(pages):
        if n < len(free):
            free[n] = page
            n += 1
        else:
            break
    return free, n
