"""The plan of the paged decode step: which pages a run takes (test data only)."""
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
