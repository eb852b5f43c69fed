"""The plan of the paged decode step (which pages a run takes) and the step in
float64 with the error that its own roundings allow, for runs of many pages
(test data and expected results only)."""
import math

import numpy as np

import _paged as P

PAGE = 64


def run_target(hq, hkv, d, fmt):
    """Runs that a call aims at: one for each wave that the chip's 1024 SIMDs hold, over kv heads and query tiles."""
    waves = {64: 3, 128: 2, 256: 1}[d]
    each = hkv * -(-(hq // hkv) // (16 if fmt == P.FP16 else 4))
    return -(-1024 * waves // each)


def units_of(d, fmt):
    return 2 if fmt == P.FP16 and d == 256 else 1


def plan(lens, hq, hkv, d, fmt):
    """The runs (sequence, first unit, end) of a call; a unit is a page, or half of one."""
    target, units = run_target(hq, hkv, d, fmt), units_of(d, fmt)
    n = [units * -(-x // PAGE) for x in lens]
    per = 1
    if sum(n) > target:
        per = -(-sum(n) // target)
        for i in range(7):
            runs = sum(-(-x // per) for x in n)
            if runs <= target or i == 6 or len(lens) >= target:
                break
            per += max(1, per * (runs - target) // target)
    out = []
    for b, x in enumerate(n):
        count = -(-x // per)
        for k in range(count):
            begin = k * (x // count) + min(k, x % count)
            out.append((b, begin, begin + x // count + (k < x % count)))
    return out


def pool_values(pool, d, fmt):
    """K and V of every record, float64 [pages, hkv, 64, d]."""
    out = np.zeros((2,) + pool.shape[:2] + (PAGE, d))
    for i in range(pool.shape[0]):
        for h in range(pool.shape[1]):
            for part in (0, 1):
                out[part, i, h] = P.read_record(pool[i, h], d, fmt, part)
    return out


def digits_of(x):
    """What four digits in base 32 make of groups of 64 query values, and the largest that the first three reach."""
    g = x.reshape(-1, 64)
    top = np.abs(g).max(1, keepdims=True)
    unit = np.exp2(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 3) / 32 ** 3
    return (np.rint(g / unit) * unit).reshape(-1), np.repeat(unit * 32 ** 3, 64, 1).reshape(-1)


def decode(q, kv, table, lens, fmt, s=None, weights=None, decay=1.0, copies=1, rounded_p=False):
    """o, lse, weights in float64 and their bounds, from the values of the records (pool_values).  The call has every
    head `copies` times.

    u = 2^-24 is a rounding in fp32; a matrix instruction's sum counts as one step of 2 u (it may cut instead of
    rounding) for each term that is not zero.
      scores   FP16: one step a channel with a query value; HIF4: sums of digits are exact, the query moves by what
               its digits leave out, one rounding for each group of 64, two for the digits, on values up to the
               digits' own (|q| and a unit more); both: the scale, twice.
      p        relative: the score's error, the rounding of the exponent (u of its binades, which are at most 16 more
               than those to the row's largest), the exponential (2 u).  In o moreover, HIF4: 2^-19 of the page's
               largest p (half a step of 32^-3 of a value of 8 or more); FP16: two halves, 2^-22, or 2^-32 of the
               row's largest p where the second one is subnormal (2^-25 beside 2^7).
      sums     HIF4: one rounding a page in o; FP16: one step a key that counts, twice (two halves).  A rescale
               multiplies by an exponential (4 u with the rounding of its argument), at most one a page; the join of
               the runs 4 u each; a lane's 16 keys, the lanes and the quotient 24 u.
      o        rounded to fp16: 2^-11, or half of 2^-24.
      lse      the logarithm of a sum of up to 2^30: 2 u of 30 binades; two roundings.
    `rounded_p`: the step with p rounded to one fp16 value (what a test's bound has to notice)."""
    u = 2.0 ** -24
    b_, hq, d = q.shape
    hkv = kv.shape[2]
    grp, root = hq // hkv, math.sqrt(d)
    o, bo = np.zeros((2, b_, hq, d))
    lse, bl = np.full((hq, b_), -np.inf), np.zeros((hq, b_))
    w = None if weights is None else weights.astype(np.float64).copy()
    bw = None if weights is None else np.abs(w) * 2.0 ** -22
    runs = plan(lens, copies * hq, copies * hkv, d, fmt)
    for b, n in enumerate(lens):
        pages = -(-n // PAGE)
        if w is not None:
            w[b, :pages] *= decay
        row = table[b, :pages]
        page = np.repeat(np.arange(pages), PAGE)[:n]
        there = ((row >= 0) & (row < kv.shape[1]))[page]
        if not there.any():
            continue
        page = page[there]
        slot = (np.arange(n) % PAGE)[there]
        mine = [r[2] - r[1] for r in runs if r[0] == b]
        steps = max(mine)
        for h in range(hq):
            x = q[b, h].astype(np.float64)
            if s is not None:
                x = (x * s[h // grp].astype(np.float64)).astype(np.float16).astype(np.float64)
            kk, vv = kv[0, row[page], h // grp, slot], kv[1, row[page], h // grp, slot]
            sc = kk @ x / root
            m = sc.max()
            e = np.exp(sc - m)
            total = e.sum()
            p = e / total
            size = np.abs(kk)
            if fmt == P.HIF4:
                y, first = digits_of(x)
                rel = size @ np.abs(x - y) / root + (d // 64 + 5) * u * (size @ (np.abs(x) + first * (x != 0))) / root
            else:
                rel = (2 * np.count_nonzero(x) + 3) * u * (size @ np.abs(x)) / root
            rel = rel + u * (math.log(2) * 16 + np.abs(sc - m)) + 2 * u
            sums = steps * 5 * u + len(mine) * 4 * u + 24 * u
            biggest = np.zeros(pages)
            np.maximum.at(biggest, page, p)
            counts = np.count_nonzero(p > 2.0 ** -60)
            moved = float(p @ rel) + sums
            used = p
            if rounded_p:
                used = (p / p.max() * 2.0 ** 14).astype(np.float16).astype(np.float64) * (p.max() / 2.0 ** 14)
            o[b, h] = used @ vv
            av = np.abs(vv)
            bo[b, h] = 1.01 * ((p * rel) @ av + float(p @ rel) * np.abs(o[b, h]) + 2 * sums * (p @ av))
            if fmt == P.HIF4:
                bo[b, h] += 2.0 ** -19 * (biggest[page] @ av)
            else:
                bo[b, h] += 2 * u * (2 * counts + 2) * (p @ av) + (2.0 ** -22 * p + 2.0 ** -32 * p.max()) @ av
            bo[b, h] += 2.0 ** -11 * (np.abs(o[b, h]) + bo[b, h]) + 2.0 ** -25
            lse[h, b] = m + math.log(total)
            bl[h, b] = 1.01 * moved + 2 * u * (30 + abs(lse[h, b]))
            if w is not None:
                per, err = np.zeros(pages), np.zeros(pages)
                np.add.at(per, page, p)
                np.add.at(err, page, p * rel)
                w[b, :pages] += copies * per
                bw[b, :pages] += copies * (1.01 * (err + per * (moved + 64 * u)) + 2.0 ** -100)
    if w is not None:
        bw += (copies * hq + 4) * u * np.abs(w)
    return o, lse, w, bo, bl, bw
