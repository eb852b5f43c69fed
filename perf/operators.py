"""Timed cases of the paged key-value cache: writing it, reading it back, attending over it and evicting from it.

Four operators of a serving loop whose cache lives in pages of 64 tokens:

  append   hifa4_paged_append: new tokens' K and V into their sequences' pages
           (one token per sequence, or chunks of a prompt), and
           hifa4_paged_gather, which reads the pages that it touched back;
  gather   hifa4_paged_gather alone: whole sequences out of the pages;
  decode   hifa4_paged_decode_fwd: one new token's attention over the pages,
           with the attention weight of each page accumulated where asked for;
  evict    hifa4_paged_evict: the pages of the least accumulated weight leave a
           sequence that holds more than its budget.

A page holds 64 tokens of every kv head, one record per head, either in HIF4
(4.5 bits a value) or in fp16.  The record is what the matrix instructions take
(`_tiles` and `_fp16_page` below spell it out), so a cache is read and written
through the operators only.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
APPEND, GATHER, DECODE, EVICT = "append", "gather", "decode", "evict"


def _case(name, kind, batch, hq, hkv, d, s, fmt="hif4", lo=0, lens=0, smooth=False, weights=False, pad=0, new=0, budget=0):
    """`lo` > 0: sequences of lengths drawn in [lo, s] from generator `lens`, else all of s; the last `pad` rows of the
    batch are empty.  `new`: tokens appended to each sequence (0: all of it)."""
    return {"name": name, "kind": kind, "batch": batch, "hq": hq, "hkv": hkv, "d": d, "s": s, "fmt": fmt, "lo": lo,
            "lens": lens, "smooth": smooth, "weights": weights, "pad": pad, "new": new, "budget": budget}


def listed():
    return [
        # one new token for each of 32 conversations of mixed lengths: what every decode step writes first
        _case("append_step_b32", APPEND, 32, 32, 8, 128, 8192, lo=300, smooth=True, new=1),
        # a batch of prompts of mixed lengths goes into the cache (the lengths of the varlen workload)
        _case("append_prompts_b16", APPEND, 16, 32, 8, 128, 2048, lo=512, smooth=True),
        # the same prompts, wide heads, into 16-bit pages
        _case("append_prompts_fp16_d256", APPEND, 16, 16, 8, 256, 2048, "fp16", lo=512),
        # a preempted conversation is read back
        _case("gather_b1_l4096", GATHER, 1, 32, 8, 128, 4096, smooth=True),
        # long conversations move to another cache
        _case("gather_varlen_b32", GATHER, 32, 32, 8, 128, 8192, lo=300, smooth=True),
        # one token of a single chat: the step's latency
        _case("decode_b1_l4096", DECODE, 1, 32, 8, 128, 4096, smooth=True),
        # one token for each of 8 long conversations: the largest cache
        _case("decode_b8_l32768", DECODE, 8, 32, 8, 128, 32768, smooth=True),
        # a serving batch of mixed lengths that keeps the weight of each page, three places of the batch empty
        _case("decode_varlen_b35_weights", DECODE, 35, 32, 8, 128, 8192, lo=300, smooth=True, weights=True, pad=3),
        # 16-bit pages, wide heads, two query heads per kv head
        _case("decode_fp16_d256_b4", DECODE, 4, 16, 8, 256, 8192, "fp16", lo=1000),
        # 16-bit pages, narrow heads, one query head per kv head, odd lengths
        _case("decode_fp16_d64_mha_b3", DECODE, 3, 12, 12, 64, 777, "fp16", lo=1),
        # long conversations are cut to a quarter of their pages
        _case("evict_b8_l32768", EVICT, 8, 32, 8, 128, 32768, budget=128),
        # a large batch of longer ones, lengths mixed
        _case("evict_varlen_b64_l131072", EVICT, 64, 32, 8, 128, 131072, lo=300, budget=256),
    ]


_MOST_BYTES = 8 * 32768 * 8 * 128 * 2 * 36 // 64          # the cache of decode_b8_l32768


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice([APPEND] * 4 + [GATHER] * 2 + [DECODE] * 8 + [EVICT] * 2)
    d = rng.choice([64, 128, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 8, 12])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 5, 8])
    fmt = rng.choice(["hif4", "hif4", "fp16"])
    smooth = fmt == "hif4" and rng.random() < 0.7
    batch = _log_int(rng, 1, 64)
    s = _log_int(rng, 1, 131072 if kind == EVICT else 32768)
    lo = max(1, s // rng.randrange(2, 17)) if batch > 1 and rng.random() < 0.6 else 0
    lens = rng.randrange(1, 1 << 20)
    new = 0
    if kind == APPEND and rng.random() < 0.6:
        new = rng.choice([1, 1, _log_int(rng, 2, 200)])
    pad = rng.choice([0, 0, 1, 2]) if kind == DECODE and batch > 3 else 0
    weights = kind == DECODE and rng.random() < 0.4
    budget = rng.randrange(1, 1 + max(2, s // PAGE)) if kind == EVICT else 0
    return _case("", kind, batch, hq, hkv, d, s, fmt, lo, lens, smooth, weights, pad, new, budget)


def draw(rng):
    while True:
        c = _draw_once(rng)
        lens = _lengths(c)
        held = sum((n + PAGE - 1) // PAGE for n in lens) * _page_bytes(c)
        values = sum(_taken(c)) * c["hkv"] * c["d"] if c["kind"] in (APPEND, GATHER) else 0
        if c["kind"] == EVICT or (held <= _MOST_BYTES and values <= 1 << 26):
            del c["name"]
            return c


# ---------------------------------------------------------------------------
# Sizes.
def _lengths(c):
    """Cached tokens of each row of the batch, the new ones included."""
    n = c["batch"] - c["pad"]
    if c["lo"] <= 0:
        lens = [c["s"]] * n
    else:
        lens = [int(x) for x in np.random.default_rng(c["lens"]).integers(c["lo"], c["s"] + 1, n)]
    return lens + [0] * c["pad"]


def _new(c):
    """Tokens that an append brings, per sequence."""
    return [min(n, c["new"]) if c["new"] else n for n in _lengths(c)]


def _starts(c):
    """First token that is read back: of an append the start of the first page that it writes to."""
    lens = _lengths(c)
    if c["kind"] == GATHER:
        return [0] * len(lens)
    return [(n - m) // PAGE * PAGE for n, m in zip(lens, _new(c))]


def _taken(c):
    """Tokens read back, per sequence."""
    return [n - a for n, a in zip(_lengths(c), _starts(c))]


def _pages(c):
    return [(n + PAGE - 1) // PAGE for n in _lengths(c)]


def _page_bytes(c):
    """Bytes of a page: K and V of 64 tokens, every kv head."""
    return c["hkv"] * PAGE * c["d"] * 2 * (36 if c["fmt"] == "hif4" else 128) // 64


def work(case):
    c = case
    lens, d, hq, hkv, b = _lengths(c), c["d"], c["hq"], c["hkv"], c["batch"]
    token = hkv * d * 2 * 2                                  # K and V of a token in fp16
    cached = token * 36 // 128 if c["fmt"] == "hif4" else token
    scales = 4 * hkv * d if c["smooth"] else 0
    if c["kind"] == DECODE:
        n = sum(lens) * cached + b * hq * (4 * d + 4) + scales + 4 * sum(_pages(c)) + 4 * b
        n += 8 * sum(_pages(c)) if c["weights"] else 0
        return {"bytes": n, "flops": 4.0 * d * hq * sum(lens)}
    if c["kind"] == EVICT:                                   # table and weights in, table, weights and freed pages out
        return {"bytes": 20 * sum(_pages(c)) + 12 * b, "flops": 0}
    out = sum(_taken(c)) * (token + cached) + 4 * sum(_pages(c))
    if c["kind"] == GATHER:
        return {"bytes": out, "flops": 0}
    moved = sum(_new(c)) * token + scales
    if c["fmt"] == "hif4":                                   # V of the last, open page is kept in fp16 beside the pages
        old = [(n - m) % PAGE if (n - m) // PAGE == (n - 1) // PAGE else 0 for n, m in zip(lens, _new(c)) if n]
        tail = [min(m, (n - 1) % PAGE + 1) for n, m in zip(lens, _new(c)) if n]
        moved += (sum(old) + sum(tail)) * token // 2
    return {"bytes": moved + out + sum(_new(c)) * cached, "flops": 0}


# ---------------------------------------------------------------------------
# HIF4 (groups of 64 values: an E6M2 base b, a halving bit per 8 and per 4 values, sign and 3-bit magnitude u per
# value; value = u b/4 2^-(E2+E3)) and the pages' records.
def _round16(x):
    """float64 to fp16, rounded once (torch goes through float32: made odd there, so that the second rounding is exact)."""
    f = x.float()
    b = f.view(torch.int32)
    b = torch.where(f.double().abs() > x.abs(), b - 1, b)
    b = torch.where(f.double() != x, b | 1, b)
    return b.view(torch.float32).half()


def _quantized(x):
    """HIF4 of float32 groups of 64 along the last axis: (u with its sign, base byte, E2 [.., 8], E3 [.., 16])."""
    a = x.abs()
    a4 = a.unflatten(-1, (16, 4)).amax(-1)
    a8 = a4.unflatten(-1, (8, 2)).amax(-1)
    top = a8.amax(-1)
    mant, ex = torch.frexp(top)                              # the smallest base that 1.75 times covers the maximum
    over = sum((mant > 7 * i / 64).int() for i in range(5, 9))
    byte = torch.where(top > 0, ((ex + 29) << 2) + 1 + over, 0)
    b = _base(byte)
    e2 = a8 <= 0.875 * b[..., None]
    e3 = a4 <= 0.875 * b[..., None] * torch.where(e2, 0.5, 1.0).repeat_interleave(2, -1)
    step = _steps(byte, e2, e3)
    u = torch.floor(a.double() / step.double() + 0.5).float()  # (borders are halves: 64 bits keep them)
    return torch.where(x < 0, -u, u), byte, e2, e3


def _base(byte):
    return torch.ldexp(1.0 + (byte & 3).float() / 4, (byte >> 2) - 31)


def _steps(byte, e2, e3):
    sh = e2.float().repeat_interleave(2, -1) + e3.float()
    return (_base(byte)[..., None] / 4 * torch.exp2(-sh)).repeat_interleave(4, -1)


def _values(x):
    """What HIF4 makes of float32 groups of 64 along the last axis."""
    u, byte, e2, e3 = _quantized(x)
    return u * _steps(byte, e2, e3)


def _pack(x):
    """HIF4 bytes of float32 tiles [.., G, 64 rows (t, n), 64 values]: codes, then metadata.

    Of a tile's row 16t + n, word w = 2k + c (values 8w to 8w + 7, value i in nibble i) goes to lane 16k + n.
    Codes [G][t/2][k][n][t%2][c], 4 bytes each.  Metadata: E3 [k][n], per lane one byte for the values 0 to 3 of each
    word and one for the values 4 to 7, bit 2t + c (two tiles' low bytes, then their high bytes, where there are two);
    E2 [k][n][G], one byte, bit 2t + c; bases [n/4][G][t][n%4], one byte."""
    u, byte, e2, e3 = _quantized(x)
    g, lead = x.shape[-3], x.shape[:-3]
    nib = u.abs().int() | ((u < 0).int() << 3)
    nib = nib.view(*lead, g, 2, 2, 16, 4, 2, 4, 2)            # G, t/2, t%2, n, k, c, byte, nibble
    code = nib[..., 0] | (nib[..., 1] << 4)
    n0 = len(lead)
    order = [n0, n0 + 1, n0 + 4, n0 + 3, n0 + 2, n0 + 5, n0 + 6]
    codes = code.permute(*range(n0), *order).reshape(*lead, -1).to(torch.uint8)
    bit = 1 << (2 * torch.arange(4, device=x.device)[:, None] + torch.arange(2, device=x.device))      # [t, c]
    e3 = e3.view(*lead, g, 4, 16, 4, 2, 2).int()              # G, t, n, k, c, half
    e3 = (e3 * bit.view(4, 1, 1, 2, 1)).sum((n0 + 1, n0 + 4))  # G, n, k, half
    e3 = e3.view(*lead, max(1, g // 2), min(2, g), 16, 4, 2).permute(*range(n0), n0 + 3, n0 + 2, n0, n0 + 4, n0 + 1)
    e2 = e2.view(*lead, g, 4, 16, 4, 2).int()
    e2 = (e2 * bit.view(4, 1, 1, 2)).sum((n0 + 1, n0 + 4)).permute(*range(n0), n0 + 2, n0 + 1, n0)      # k, n, G
    base = byte.view(*lead, g, 4, 4, 4).permute(*range(n0), n0 + 2, n0, n0 + 1, n0 + 3)
    meta = [m.reshape(*lead, -1).to(torch.uint8) for m in (e3, e2, base)]
    return torch.cat([codes] + meta, -1)


def _tiles(rec, g):
    """float32 tiles [.., G, 64 rows, 64 values] of HIF4 bytes [.., 2304 G]: what _pack wrote."""
    lead, n0 = rec.shape[:-1], rec.dim() - 1
    code = rec[..., :2048 * g].reshape(*lead, g, 2, 4, 16, 2, 2, 4)
    code = code.permute(*range(n0), n0, n0 + 1, n0 + 4, n0 + 3, n0 + 2, n0 + 5, n0 + 6).reshape(*lead, g, 64, 32)
    nib = torch.stack([code & 15, code >> 4], -1).reshape(*lead, g, 64, 64)
    u = torch.where(nib >= 8, -(nib & 7).float(), (nib & 7).float())
    at = 2 * torch.arange(4, device=rec.device)[:, None] + torch.arange(2, device=rec.device)            # [t, c]
    e3 = rec[..., 2048 * g:2176 * g].reshape(*lead, 4, 16, max(1, g // 2), 2, min(2, g))
    e3 = e3.permute(*range(n0), n0 + 2, n0 + 4, n0 + 1, n0, n0 + 3).reshape(*lead, g, 1, 16, 4, 1, 2)    # G, n, k, half
    e3 = ((e3 >> at.view(4, 1, 1, 2, 1).to(torch.uint8)) & 1).reshape(*lead, g, 64, 16)
    e2 = rec[..., 2176 * g:2240 * g].reshape(*lead, 4, 16, g)
    e2 = e2.permute(*range(n0), n0 + 2, n0 + 1, n0).reshape(*lead, g, 1, 16, 4, 1)
    e2 = ((e2 >> at.view(4, 1, 1, 2).to(torch.uint8)) & 1).reshape(*lead, g, 64, 8)
    base = rec[..., 2240 * g:].reshape(*lead, 4, g, 4, 4).permute(*range(n0), n0 + 1, n0 + 2, n0, n0 + 3)
    return u * _steps(base.reshape(*lead, g, 64).int(), e2, e3)


def _key_rows(x):
    """[.., 64 keys, D] as tiles [.., G, 64 rows, 64 channels]: key 16a + 4t + b is row 16t + 4a + b."""
    x = x.unflatten(-2, (4, 4, 4)).transpose(-4, -3).flatten(-4, -2)
    return x.unflatten(-1, (-1, 64)).transpose(-3, -2)


def _rows_keys(x):
    x = x.transpose(-3, -2).flatten(-2)
    return x.unflatten(-2, (4, 4, 4)).transpose(-4, -3).flatten(-4, -2)


def _hif4_page(k, v):
    """The record [.., 4608 G] of a page's K and V [.., 64, D] (float32): K's tiles, then V's (rows are channels)."""
    vt = v.transpose(-2, -1).unflatten(-2, (-1, 64))
    return torch.cat([_pack(_key_rows(k).contiguous()), _pack(vt.contiguous())], -1)


def _fp16_page(k, v):
    """The record [.., 256 D] of a page's K and V [.., 64, D] (fp16): K [t][D/32][k][n][8 channels] for the keys of
    _key_rows, V [D/16][c][k][16 channels][8 keys], the keys 16k + 8c and up."""
    lead, d, n0 = k.shape[:-2], k.shape[-1], k.dim() - 2
    kr = _rows16(k).view(*lead, 4, 16, d // 32, 4, 8).permute(*range(n0), n0, n0 + 2, n0 + 3, n0 + 1, n0 + 4)
    vr = v.reshape(*lead, 4, 2, 8, d // 16, 16).permute(*range(n0), n0 + 3, n0 + 1, n0, n0 + 4, n0 + 2)
    return torch.cat([kr.reshape(*lead, -1), vr.reshape(*lead, -1)], -1).view(torch.uint8)


def _rows16(x):
    return x.unflatten(-2, (4, 4, 4)).transpose(-4, -3).flatten(-4, -2)


def _page_values(c, rec):
    """K and V [.., 64, D] in float32 of pages' records [.., bytes]."""
    d, lead, n0 = c["d"], rec.shape[:-1], rec.dim() - 1
    if c["fmt"] == "hif4":
        g = d // 64
        half = 2304 * g
        v = _tiles(rec[..., half:], g).flatten(-3, -2).transpose(-2, -1)
        return _rows_keys(_tiles(rec[..., :half], g)), v
    x = rec.view(torch.float16).float()
    k = x[..., :64 * d].reshape(*lead, 4, d // 32, 4, 16, 8).permute(*range(n0), n0, n0 + 3, n0 + 1, n0 + 2, n0 + 4)
    v = x[..., 64 * d:].reshape(*lead, d // 16, 2, 4, 16, 8).permute(*range(n0), n0 + 2, n0 + 1, n0 + 4, n0, n0 + 3)
    return _rows16(k.reshape(*lead, 64, d)), v.reshape(*lead, 64, d)


# ---------------------------------------------------------------------------
# Inputs.
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _gain(c, dev):
    """[Hkv, D] factors of the key channels: the model's amplified channels (x16), ones elsewhere."""
    g = np.random.default_rng(4242)
    gain = np.ones((c["hkv"], c["d"]), np.float32)
    if c["smooth"]:
        for h in range(c["hkv"]):
            gain[h, g.choice(c["d"], c["d"] // 32, replace=False)] = 16.0
    return torch.from_numpy(gain).to(dev)


def _scales(c, dev):
    """Smooth-QK scales [Hkv, D] of the model, or None: about the root of the keys' amplification."""
    if not c["smooth"]:
        return None
    jitter = torch.from_numpy(np.random.default_rng(77).uniform(0.9, 1.1, (c["hkv"], c["d"])).astype(np.float32))
    return _gain(c, dev).sqrt() * jitter.to(dev)


def _ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _cu(counts, dev):
    return _ints([0] + [int(x) for x in np.cumsum(counts)], dev)


def prepare(case, seed):
    c, dev = case, _device()
    gen = torch.Generator(device=dev).manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    lens, pages = _lengths(c), _pages(c)
    b, d, hq, hkv = c["batch"], c["d"], c["hq"], c["hkv"]
    total, most = sum(pages), max(pages)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    # the sequences' pages are spread over the pool; places behind a sequence's end hold no page
    free = torch.randperm(total + 1, generator=gen, device=dev).int()
    count = torch.tensor(pages, device=dev)
    column = torch.arange(most, device=dev)
    used = column < count[:, None]
    first = torch.cumsum(count, 0) - count
    table = torch.where(used, free[(first[:, None] + column).clamp(max=total)], -1).contiguous()
    st = {"case": c, "table": table, "lens": _ints(lens, dev)}
    if c["kind"] == EVICT:
        # weights of a few hundred steps: the first page and the last ones draw most, the rest by a long-tailed law
        w = torch.exp(1.5 * normal(b, most))
        w[:, 0] += 40.0
        w += torch.where(column >= count[:, None] - 2, 20.0, 0.0)
        st.update(w=torch.where(used, w, 0.0), out_table=torch.empty_like(table), out_lens=torch.empty_like(st["lens"]),
                  out_w=torch.empty_like(w), freed=torch.empty_like(table), num_freed=torch.empty_like(st["lens"]))
        return st
    s = st["s"] = _scales(c, dev)
    gain = _gain(c, dev)
    bytes_ = _page_bytes(c) // hkv
    pool = torch.empty((total + 1, hkv, bytes_), dtype=torch.uint8, device=dev)
    for at in range(0, total + 1, 512):
        n = min(512, total + 1 - at)
        k, v = normal(n, hkv, PAGE, d) * gain[:, None], normal(n, hkv, PAGE, d)
        k = (k if s is None else k / s[:, None]).half()
        pool[at:at + n] = _hif4_page(k.float(), v.half().float()) if c["fmt"] == "hif4" else _fp16_page(k, v.half())
    st["pool"] = pool
    if c["kind"] == DECODE:
        st["q"] = normal(b, hq, d).half()
        if c["weights"]:
            st["w"] = torch.where(used, torch.exp(normal(b, most)), 0.0)
            st["out_w"] = st["w"].clone()
    else:
        taken = _taken(c)
        st.update(starts=_ints(_starts(c), dev), cu_out=_cu(taken, dev), total=sum(taken), most=max(taken))
        if c["kind"] == APPEND:
            new = _new(c)
            t = sum(new)
            st.update(k=(normal(t, hkv, d) * gain).half(), v=normal(t, hkv, d).half(), cu_new=_cu(new, dev), most_new=max(new))
            if c["fmt"] == "hif4":
                st["tail0"] = normal(b, PAGE, hkv, d).half()
                st["tail"] = st["tail0"].clone()
    if own:
        import paper_2607_04302_amd as h4
        st["cache"] = h4.PagedCache(pool, table, st["lens"], d,
                                    h4.OPERANDS_HIF4 if c["fmt"] == "hif4" else h4.OPERANDS_FP16, v_tail=st.get("tail"))
    return st


# ---------------------------------------------------------------------------
# The plain forms.
def _sequence_of(cu, total):
    """Row of the batch, and place within its run, of each of the `total` tokens that cu counts."""
    at = torch.arange(total, device=cu.device)
    row = torch.searchsorted(cu[1:].long().contiguous(), at, right=True)
    return row, at - cu[row]


def _plain_gather(c, x):
    row, at = _sequence_of(x["cu_out"], x["total"])
    pos = x["starts"][row] + at
    k, v = _page_values(c, x["pool"])                         # [pages, Hkv, 64, D]
    page = x["table"][row, pos // PAGE].long()
    return k[page, :, pos % PAGE].half(), v[page, :, pos % PAGE].half()


def _plain_append(c, x):
    """What the pages hold of the tokens that are read back, once the new tokens are in."""
    row, at = _sequence_of(x["cu_out"], x["total"])
    pos = x["starts"][row] + at
    count = x["cu_new"][1:] - x["cu_new"][:-1]
    index = x["cu_new"][row] + pos - (x["lens"] - count)[row]  # the new token at this place; negative: an old one
    fresh = pos >= (x["lens"] - count)[row]
    index = torch.where(fresh, index, 0)
    page = x["table"][row, pos // PAGE].long()
    records, inverse = torch.unique(page, return_inverse=True)
    old_k, old_v = _page_values(c, x["pool"][records])
    old_k, old_v = old_k[inverse, :, pos % PAGE], old_v[inverse, :, pos % PAGE]
    keep = fresh[:, None, None]
    if c["fmt"] == "fp16":
        return {"k": torch.where(keep, x["k"][index], old_k.half()), "v": torch.where(keep, x["v"][index], old_v.half())}
    k = x["k"] if x["s"] is None else _round16(x["k"].double() / x["s"].double())
    k = _values(k.float().unflatten(-1, (-1, 64))).flatten(-2)[index]
    v = torch.where(keep, x["v"][index], x["tail0"][row, pos % PAGE])
    nb = (x["most"] + PAGE - 1) // PAGE
    blocks = torch.zeros((c["batch"], nb * PAGE, c["hkv"], c["d"]), device=v.device)
    blocks[row, at] = v.float()
    vq = _values(blocks.unflatten(1, (nb, PAGE)).transpose(2, 4).contiguous()).transpose(2, 4).flatten(1, 2)
    tail = x["tail0"].clone()
    last = (pos // PAGE == ((x["lens"] - 1) // PAGE)[row]) & fresh
    tail[row[last], pos[last] % PAGE] = v[last]
    return {"k": torch.where(keep, k.half(), old_k.half()), "v": vq[row, at].half(), "tail": tail}


def _plain_decode(c, x):
    b, d, hq, hkv = c["batch"], c["d"], c["hq"], c["hkv"]
    k, v = _page_values(c, x["pool"])
    n = x["table"].shape[1] * PAGE
    at = x["table"].clamp(min=0).long()
    k = k[at].transpose(1, 2).reshape(b, hkv, n, d)
    v = v[at].transpose(1, 2).reshape(b, hkv, n, d)
    q = x["q"].view(b, hkv, hq // hkv, d)
    q = (q if x["s"] is None else _round16(q.double() * x["s"].double()[:, None])).float()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    hidden = torch.arange(n, device=s.device) >= x["lens"][:, None, None, None]
    s = torch.where(hidden, -math.inf, s)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    p = p / torch.where(l > 0, l, 1.0)
    out = {"o": torch.matmul(p, torch.where(hidden.transpose(2, 3), 0.0, v)).view(b, hq, d).half(),
           "lse": (m + torch.log(l)).view(b, hq).t().contiguous()}
    if c["weights"]:
        w = p.view(b, hq, n // PAGE, PAGE).sum((1, 3))
        used = torch.arange(n // PAGE, device=s.device) * PAGE < x["lens"][:, None]
        out["weights"] = torch.where(used, 0.875 * x["w"] + w, x["w"])
    return out


def _evict_rule(c):
    """(budget, first pages kept, last pages kept) of the case."""
    budget = c["budget"]
    return budget, min(1, budget - 1), max(1, min(2, budget - 1))


def _plain_evict(c, x):
    budget, first, last = _evict_rule(c)
    table, lens, w = x["table"], x["lens"], x["w"]
    column = torch.arange(table.shape[1], device=w.device)
    pages = ((lens + PAGE - 1) // PAGE)[:, None]
    used = column < pages
    rank = torch.where((column < first) | (column >= pages - last), math.inf, w)
    rank = torch.where(used, rank, -math.inf)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices      # ties: the lowest place first
    place = torch.argsort(order, dim=1)
    kept = used & (place < budget)
    gone = used & ~kept
    num = gone.sum(1).int()

    def moved(x, which, fill):
        to = torch.where(which, torch.cumsum(which, 1) - 1, table.shape[1])
        out = torch.full((table.shape[0], table.shape[1] + 1), fill, dtype=x.dtype, device=x.device)
        return out.scatter(1, to, torch.where(which, x, fill))[:, :-1].contiguous()

    return {"table": moved(table, kept, -1), "lens": lens - PAGE * num, "weights": moved(w, kept, 0.0),
            "freed": moved(table, gone, -1), "num_freed": num}


def run(state):
    c, x = state["case"], state
    if not own:
        if c["kind"] == GATHER:
            k, v = _plain_gather(c, x)
            return {"k": k, "v": v}
        return {APPEND: _plain_append, DECODE: _plain_decode, EVICT: _plain_evict}[c["kind"]](c, x)
    import paper_2607_04302_amd as h4
    if c["kind"] == EVICT:
        budget, first, last = _evict_rule(c)
        h4.hifa4_paged_evict(x["table"], x["lens"], x["w"], budget, first, last, out_table=x["out_table"],
                             out_lens=x["out_lens"], out_weights=x["out_w"], freed=x["freed"], num_freed=x["num_freed"])
        return {"table": x["out_table"], "lens": x["out_lens"], "weights": x["out_w"], "freed": x["freed"],
                "num_freed": x["num_freed"]}
    cache = x["cache"]
    if c["kind"] == DECODE:
        if not c["weights"]:
            o, lse = h4.hifa4_paged_decode_fwd(cache, x["q"], x["s"])
            return {"o": o, "lse": lse}
        o, lse = h4.hifa4_paged_decode_fwd(cache, x["q"], x["s"], page_weights=x["w"], decay=0.875, weights_out=x["out_w"])
        return {"o": o, "lse": lse, "weights": x["out_w"]}
    out = {}
    if c["kind"] == APPEND:
        if "tail" in x:
            if c["new"] > 1:      # chunks that cross a page overwrite the rows that the next pass starts from
                x["tail"].copy_(x["tail0"])
            out["tail"] = x["tail"]
        h4.hifa4_paged_append(cache, x["k"], x["v"], x["s"], cu_new=x["cu_new"], max_new=x["most_new"])
    out["k"], out["v"] = h4.hifa4_paged_gather(cache, x["cu_out"], x["total"], max_tokens=x["most"], starts=x["starts"])
    return out


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions: every value looked up in the page's bytes by its own address.
def _addresses(d, dev):
    """Of each (key, channel) of a HIF4 record: byte and shift of the code, byte and bit of E2 and E3, byte of the base;
    K, then V."""
    g = d // 64
    key, ch = np.meshgrid(np.arange(64), np.arange(d), indexing="ij")
    out = []
    for part in (0, 1):
        if part == 0:
            row, tile, elem = 16 * (key // 4 % 4) + 4 * (key // 16) + key % 4, ch // 64, ch % 64
        else:
            row, tile, elem = ch % 64, ch // 64, key
        t, n, word, i = row // 16, row % 16, elem // 8, elem % 8
        lane, bit, o = 16 * (word // 2) + n, 2 * t + word % 2, 2304 * g * part
        code = o + 2048 * tile + 1024 * (t // 2) + 16 * lane + 8 * (t % 2) + 4 * (word % 2) + i // 2
        e3 = o + 2048 * g + 2 * g * lane + (i // 4 if g == 1 else 4 * (tile // 2) + 2 * (i // 4) + tile % 2)
        e2 = o + 2176 * g + g * lane + tile
        base = o + 2240 * g + 16 * g * (n // 4) + 16 * tile + 4 * t + n % 4
        out.append([torch.from_numpy(a.reshape(-1).astype(np.int64)).to(dev) for a in (code, 4 * (i % 2), e2, e3, bit, base)])
    return out


def _addresses16(d, dev):
    key, ch = np.meshgrid(np.arange(64), np.arange(d), indexing="ij")
    row = 16 * (key // 4 % 4) + 4 * (key // 16) + key % 4
    k = (((row // 16) * (d // 32) + ch // 32) * 4 + ch // 8 % 4) * 128 + row % 16 * 8 + ch % 8
    v = 64 * d + (((ch // 16) * 2 + key // 8 % 2) * 4 + key // 16) * 128 + ch % 16 * 8 + key % 8
    return [torch.from_numpy(a.reshape(-1).astype(np.int64)).to(dev) for a in (k, v)]


def _look_up(c, rec):
    """K and V [.., 64, D] in float64 of records [.., bytes]."""
    out, d, dev = [], c["d"], rec.device
    if c["fmt"] == "fp16":
        x = rec.view(torch.float16)
        return [x[..., a].double().view(*rec.shape[:-1], 64, d) for a in _addresses16(d, dev)]
    nibble = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, 0, -1, -2, -3, -4, -5, -6, -7], dtype=torch.float64, device=dev)
    e6m2 = torch.tensor([(4 + i % 4) * 2.0 ** (i // 4 - 35) for i in range(256)], dtype=torch.float64, device=dev)
    for code, shift, e2, e3, bit, base in _addresses(d, dev):
        u = nibble[(rec[..., code].long() >> shift) & 15]
        sh = ((rec[..., e2].long() >> bit) & 1) + ((rec[..., e3].long() >> bit) & 1)
        out.append((u * e6m2[rec[..., base].long()] * torch.exp2(-sh.double())).view(*rec.shape[:-1], 64, d))
    return out


def _fp16_of(x):
    """float64 to fp16, rounded once."""
    return torch.from_numpy(x.cpu().numpy().astype(np.float16)).to(x.device)


def _hif4_of(x):
    """HIF4 of float64 groups of 64 along the last axis."""
    dev, parts = x.device, []
    table = torch.tensor([(4 + i % 4) * 2.0 ** (i // 4 - 33) for i in range(256)], dtype=torch.float64, device=dev)
    for y in x.reshape(-1, 64).split(1 << 20):
        b = table[torch.searchsorted(1.75 * table, y.abs().amax(1))][:, None, None, None]
        y = y.view(-1, 8, 2, 4)
        halved = torch.where(y.abs().amax((2, 3), keepdim=True) <= 0.875 * b, b / 2, b)
        step = torch.where(y.abs().amax(3, keepdim=True) <= 0.875 * halved, halved / 2, halved) / 4
        parts.append((torch.sign(y) * torch.floor(y.abs() / step + 0.5) * step).view(-1, 64))
    return torch.cat(parts).view(x.shape)


def _exact_cache(c, x):
    ks, vs, tails = [], [], []
    starts, lens, new = _starts(c), _lengths(c), _new(c)
    hif4 = c["fmt"] == "hif4"
    at = 0
    for b, n in enumerate(lens):
        pages = x["table"][b, starts[b] // PAGE:(n + PAGE - 1) // PAGE].long()
        k, v = [a.transpose(1, 2).flatten(0, 1)[:n - starts[b]] for a in _look_up(c, x["pool"][pages])]   # [tokens, Hkv, D]
        if c["kind"] == APPEND:
            m = new[b]
            nk, nv = x["k"][at:at + m], x["v"][at:at + m].double()
            at += m
            old = n - m - starts[b]
            if not hif4:
                k, v = torch.cat([k[:old], nk.double()]), torch.cat([v[:old], nv])
            else:
                nk = nk.double() if x["s"] is None else _fp16_of(nk.double() / x["s"].double()).double()
                k = torch.cat([k[:old], _hif4_of(nk.unflatten(-1, (-1, 64))).flatten(-2)])
                v = torch.cat([x["tail0"][b, :old].double(), nv])
                tail = x["tail0"][b].double()
                r = (n - 1) % PAGE + 1
                if m >= r:
                    tail[:r] = nv[m - r:]
                else:
                    tail[r - m:r] = nv
                tails.append(tail)
                full = torch.zeros(((len(v) + PAGE - 1) // PAGE * PAGE, c["hkv"], c["d"]), dtype=torch.float64, device=v.device)
                full[:len(v)] = v
                full = full.view(-1, PAGE, c["hkv"], c["d"]).permute(0, 2, 3, 1)
                v = _hif4_of(full).permute(0, 3, 1, 2).flatten(0, 1)[:len(v)]
        ks.append(k)
        vs.append(v)
    out = {"k": torch.cat(ks), "v": torch.cat(vs)}
    if tails:
        out["tail"] = torch.stack(tails)
    return out


def _exact_decode(c, x):
    b, d, hq, hkv = c["batch"], c["d"], c["hq"], c["hkv"]
    dev = x["q"].device
    o = torch.zeros((b, hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((hq, b), -math.inf, dtype=torch.float64, device=dev)
    w = x["w"].double() if c["weights"] else None
    for i, n in enumerate(_lengths(c)):
        if not n:
            continue
        at = x["table"][i, :(n + PAGE - 1) // PAGE].long()
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            k, v = [a.flatten(0, 1)[:n] for a in _look_up(c, x["pool"][at, h])]
            q = x["q"][i, heads].double()
            if x["s"] is not None:
                q = _fp16_of(q * x["s"][h].double()).double()
            s = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
            lse[heads, i] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[heads, i][:, None])
            o[i, heads] = torch.mm(p, v)
            if w is not None:
                full = torch.zeros((hq // hkv, len(at) * PAGE), dtype=torch.float64, device=dev)
                full[:, :n] = p
                w[i, :len(at)] = w[i, :len(at)] * (0.875 if h == 0 else 1.0) + full.view(-1, len(at), PAGE).sum((0, 2))
    return {"o": o, "lse": lse, **({} if w is None else {"weights": w})}


def _exact_evict(c, x):
    budget, first, last = _evict_rule(c)
    table, w = x["table"].cpu().numpy(), x["w"].cpu().numpy().astype(np.float64)
    out = {"table": np.full_like(table, -1), "lens": np.array(_lengths(c), np.int32), "weights": np.zeros_like(w),
           "freed": np.full_like(table, -1), "num_freed": np.zeros(len(table), np.int32)}
    for b, n in enumerate(_pages(c)):
        middle = sorted(range(first, n - last), key=lambda j: (-w[b, j], j)) if n > budget else []
        gone = sorted(middle[budget - first - last:])
        kept = [j for j in range(n) if j not in set(gone)]
        out["table"][b, :len(kept)], out["weights"][b, :len(kept)] = table[b, kept], w[b, kept]
        out["freed"][b, :len(gone)], out["num_freed"][b] = table[b, gone], len(gone)
        out["lens"][b] -= PAGE * len(gone)
    return {k: torch.from_numpy(v) for k, v in out.items()}


def exact(case, seed):
    c = case
    x = prepare(c, seed)
    return {APPEND: _exact_cache, GATHER: _exact_cache, DECODE: _exact_decode, EVICT: _exact_evict}[c["kind"]](c, x)
