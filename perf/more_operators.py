"""Timed cases of a serving step around the paged cache: its tables, its positions and the attention of its new tokens.

Five calls that a serving loop makes beside those of the paged cache (pages of 64 tokens out of one pool):

  extend   hifa4_paged_extend: each sequence gets the pages of its new tokens
           from a stack of free ones; prefix sums, positions and slots of the
           new tokens come out;
  release  hifa4_paged_release: pages go back on the stack;
  rope     hifa4_rope: rotary positions of the new tokens' q and k, as the
           projection leaves them (one row of q, k and v per token);
  chunk    hifa4_paged_chunk_fwd: the attention of each sequence's last tokens
           (a chunk of a prompt, a few drafted tokens, one token) over its pages.

A page holds 64 tokens of every kv head, one record per head, either in HIF4
(4.5 bits a value) or in fp16.  The record is what the matrix instructions take
(`_tiles` and `_page16` below spell it out).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
EXTEND, RELEASE, ROPE, CHUNK = "extend", "release", "rope", "chunk"


def _tables(name, kind, batch, s, lo=0, lens=0, new=1, evicted=False):
    """`batch` sequences of lengths drawn in [lo, s] from generator `lens` (lo = 0: all of s), the new tokens included;
    `new` tokens of each are new (0: all).  `evicted`: sequences that have lost pages, whose positions run ahead."""
    return {"name": name, "kind": kind, "batch": batch, "s": s, "lo": lo, "lens": lens, "new": new, "evicted": evicted}


def _rope(name, tokens, hq, hkv, d, rot, interleaved=False, scale="none", factor=1.0, far=32768, transposed=False):
    """Tokens at positions up to `far`; `rot` of the head's `d` channels are rotated."""
    return {"name": name, "kind": ROPE, "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
            "interleaved": interleaved, "scale": scale, "factor": factor, "far": far, "transposed": transposed}


def _chunk(name, batch, hq, hkv, d, s, new, fmt="hif4", lo=0, lens=0, smooth=False, mixed=False, pad=0):
    """Lengths as for _tables; with `mixed` every eighth sequence has `new` new tokens and the others one; the last `pad`
    rows of the batch are empty."""
    return {"name": name, "kind": CHUNK, "batch": batch, "hq": hq, "hkv": hkv, "d": d, "s": s, "new": new, "fmt": fmt,
            "lo": lo, "lens": lens, "smooth": smooth, "mixed": mixed, "pad": pad}


def listed():
    return [
        # one token more for each of 32 conversations of mixed lengths: before every decode step
        _tables("extend_step_b32", EXTEND, 32, 8192, lo=300),
        # many prompts arrive at once and get all of their pages
        _tables("extend_prompts_b64", EXTEND, 64, 32768, lo=300, new=0),
        # a batch of conversations ends
        _tables("release_b32", RELEASE, 32, 8192, lo=300, new=0),
        # a large batch of long ones, some of them cut back only
        _tables("release_b64_l131072", RELEASE, 64, 131072, lo=300, new=40000),
        # positions of one decode step of 32 conversations
        _rope("rope_step_t32", 32, 32, 8, 128, 128),
        # a prompt, neighbouring channels paired, frequencies stretched by parts for a longer context
        _rope("rope_prompt_t8192", 8192, 32, 8, 128, 128, interleaved=True, scale="parts", factor=4.0, far=131072),
        # wide heads of which a quarter is rotated, a batch of prompts of odd total length
        _rope("rope_part_t20011_d256", 20011, 16, 8, 256, 64, scale="linear", factor=2.0),
        # 5 drafted tokens of each of 32 conversations are checked
        _chunk("chunk_draft_b32", 32, 32, 8, 128, 8192, 5, lo=300, smooth=True),
        # a serving batch: most conversations bring one token, a few a chunk of their prompt, three rows empty
        _chunk("chunk_mixed_b35", 35, 32, 8, 128, 8192, 300, lo=300, smooth=True, mixed=True, pad=3),
        # a batch of prompts of mixed lengths from their first token on
        _chunk("chunk_prompts_b16", 16, 32, 8, 128, 2048, 0, lo=512, smooth=True),
        # 16-bit pages, wide heads, two query heads per kv head, odd lengths
        _chunk("chunk_fp16_d256_b4", 4, 16, 8, 256, 8192, 201, "fp16", lo=1000),
        # the last 2048 tokens of a long document: the largest
        _chunk("chunk_long_b1_l32768", 1, 32, 8, 128, 32768, 2048, smooth=True),
    ]


_MOST_FLOPS = 4.0 * 128 * 32 * 2048 * (32768 - 1024)      # chunk_long_b1_l32768
_MOST_BYTES = 8 * 32768 * 8 * 128 * 2 * 36 // 64          # of a cache
_MOST_VALUES = 20011 * 24 * 256                           # rope_part_t20011_d256


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice([EXTEND, RELEASE] + [ROPE] * 2 + [CHUNK] * 6)
    batch = _log_int(rng, 1, 64)
    lens = rng.randrange(1, 1 << 20)
    if kind in (EXTEND, RELEASE):
        s = _log_int(rng, 1, 131072 if kind == RELEASE else 32768)
        lo = max(1, s // rng.randrange(2, 17)) if rng.random() < 0.6 else 0
        new = rng.choice([0, 0, 1, _log_int(rng, 1, s)])
        return _tables("", kind, batch, s, lo, lens, new, kind == EXTEND and rng.random() < 0.3)
    d = rng.choice([64, 128, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 8, 12])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 5, 8])
    if kind == ROPE:
        rot = rng.choice([d, d, d // 2, d // 4, 8 * rng.randrange(1, d // 8 + 1)])
        scale = rng.choice(["none", "none", "linear", "ntk", "parts"]) if rot > 2 else "none"
        return _rope("", _log_int(rng, 1, 32768), hq, hkv, d, rot, rng.random() < 0.4, scale,
                     1.0 if scale == "none" else rng.choice([2.0, 4.0, 8.0]), _log_int(rng, 1, 1 << 20), rng.random() < 0.2)
    fmt = rng.choice(["hif4", "hif4", "fp16"])
    s = _log_int(rng, 1, 32768)
    lo = max(1, s // rng.randrange(2, 17)) if batch > 1 and rng.random() < 0.6 else 0
    new = rng.choice([0, 1, rng.randrange(2, 9), _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)])
    return _chunk("", batch, hq, hkv, d, s, new, fmt, lo, lens, fmt == "hif4" and rng.random() < 0.7, rng.random() < 0.25,
                  rng.choice([0, 0, 1, 2]) if batch > 3 else 0)


def draw(rng):
    while True:
        c = _draw_once(rng)
        if c["kind"] == ROPE:
            fits = c["tokens"] * (c["hq"] + c["hkv"]) * c["d"] <= _MOST_VALUES
        elif c["kind"] == CHUNK:
            fits = sum(_pages(c)) * _page_bytes(c) <= _MOST_BYTES and work(c)["flops"] <= _MOST_FLOPS
        else:
            fits = True
        if fits:
            del c["name"]
            return c


# ---------------------------------------------------------------------------
# Sizes.
def _lengths(c):
    """Tokens of each row of the batch, the new ones included."""
    pad = c.get("pad", 0)
    n = c["batch"] - pad
    if c["lo"] <= 0:
        lens = [c["s"]] * n
    else:
        lens = [int(x) for x in np.random.default_rng(c["lens"]).integers(c["lo"], c["s"] + 1, n)]
    return lens + [0] * pad


def _new(c):
    """New tokens of each row."""
    out = []
    for i, n in enumerate(_lengths(c)):
        m = c["new"] if c["new"] else n
        out.append(min(n, 1 if c.get("mixed") and i % 8 else m))
    return out


def _pages(c):
    return [(n + PAGE - 1) // PAGE for n in _lengths(c)]


def _old_pages(c):
    return [(n - m + PAGE - 1) // PAGE for n, m in zip(_lengths(c), _new(c))]


def _page_bytes(c):
    """Bytes of a page: K and V of 64 tokens, every kv head."""
    return c["hkv"] * PAGE * c["d"] * 2 * (36 if c["fmt"] == "hif4" else 128) // 64


def work(case):
    c = case
    if c["kind"] == ROPE:                                     # q and k in and out, a position per token
        return {"bytes": c["tokens"] * (4 * (c["hq"] + c["hkv"]) * c["d"] + 4),
                "flops": 3.0 * c["tokens"] * (c["hq"] + c["hkv"]) * c["rot"]}
    lens, new, b = _lengths(c), _new(c), c["batch"]
    moved = sum(_pages(c)) - sum(_old_pages(c))
    if c["kind"] == EXTEND:     # lengths and counts in, lengths and sums out, the pages, positions and slots
        return {"bytes": 16 * b + (4 * b if c["evicted"] else 0) + 8 * moved + 12 * sum(new), "flops": 0}
    if c["kind"] == RELEASE:
        return {"bytes": 8 * b + 8 * moved, "flops": 0}
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    token = hkv * d * 2 * 2                                   # K and V of a token in fp16
    cached = token * 36 // 128 if c["fmt"] == "hif4" else token
    n = sum(x for x, m in zip(lens, new) if m) * cached + sum(new) * hq * (4 * d + 4) + (4 * hkv * d if c["smooth"] else 0)
    seen = sum(m * x - m * (m - 1) // 2 for x, m in zip(lens, new))
    return {"bytes": n + 4 * sum(_pages(c)) + 8 * b, "flops": 4.0 * d * hq * seen}


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


def _base(byte):
    return torch.ldexp(1.0 + (byte & 3).float() / 4, (byte >> 2) - 31)


def _steps(byte, e2, e3):
    sh = e2.float().repeat_interleave(2, -1) + e3.float()
    return (_base(byte)[..., None] / 4 * torch.exp2(-sh)).repeat_interleave(4, -1)


def _pack(x):
    """HIF4 bytes of float32 tiles [.., G, 64 rows (t, n), 64 values]: codes, then metadata.

    Of a tile's row 16t + n, word w = 2k + c (values 8w to 8w + 7, value i in nibble i) goes to lane 16k + n.
    Codes [G][t/2][k][n][t%2][c], 4 bytes each.  Metadata: E3 [k][n], per lane one byte for the values 0 to 3 of each
    word and one for the values 4 to 7, bit 2t + c (two tiles' low bytes, then their high bytes, where there are two);
    E2 [k][n][G], one byte, bit 2t + c; bases [n/4][G][t][n%4], one byte."""
    a4 = x.abs().unflatten(-1, (16, 4)).amax(-1)
    a8 = a4.unflatten(-1, (8, 2)).amax(-1)
    mant, ex = torch.frexp(a8.amax(-1))                      # the smallest base that 1.75 times covers the maximum
    over = sum((mant > 7 * i / 64).int() for i in range(5, 9))
    byte = torch.where(mant > 0, ((ex + 29) << 2) + 1 + over, 0)
    b = _base(byte)
    e2 = a8 <= 0.875 * b[..., None]
    e3 = a4 <= 0.875 * b[..., None] * torch.where(e2, 0.5, 1.0).repeat_interleave(2, -1)
    u = torch.floor(x.abs().double() / _steps(byte, e2, e3).double() + 0.5).int()
    g, lead = x.shape[-3], x.shape[:-3]
    nib = u | (((x < 0) & (u > 0)).int() << 3)
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


def _key_order(x):
    """[.., 64 keys, D] with key 16a + 4t + b in row 16t + 4a + b, or back."""
    return x.unflatten(-2, (4, 4, 4)).transpose(-4, -3).flatten(-4, -2)


def _page4(k, v):
    """The HIF4 record [.., 4608 G] of a page's K and V [.., 64, D] (float32): K's tiles, then V's (rows are channels)."""
    kt = _key_order(k).unflatten(-1, (-1, 64)).transpose(-3, -2).contiguous()
    vt = v.transpose(-2, -1).unflatten(-2, (-1, 64)).contiguous()
    return torch.cat([_pack(kt), _pack(vt)], -1)


def _page16(k, v):
    """The fp16 record [.., 256 D] of a page's K and V [.., 64, D]: K [t][D/32][k][n][8 channels] in the order of
    _key_order, V [D/16][c][k][16 channels][8 keys], the keys 16k + 8c and up."""
    lead, d, n0 = k.shape[:-2], k.shape[-1], k.dim() - 2
    kr = _key_order(k).view(*lead, 4, 16, d // 32, 4, 8).permute(*range(n0), n0, n0 + 2, n0 + 3, n0 + 1, n0 + 4)
    vr = v.reshape(*lead, 4, 2, 8, d // 16, 16).permute(*range(n0), n0 + 3, n0 + 1, n0, n0 + 4, n0 + 2)
    return torch.cat([kr.reshape(*lead, -1), vr.reshape(*lead, -1)], -1).view(torch.uint8)


def _page_values(c, rec):
    """K and V [.., 64, D] in float32 of pages' records [.., bytes]."""
    d, lead, n0 = c["d"], rec.shape[:-1], rec.dim() - 1
    if c["fmt"] == "hif4":
        g = d // 64
        half = 2304 * g
        v = _tiles(rec[..., half:], g).flatten(-3, -2).transpose(-2, -1)
        return _key_order(_tiles(rec[..., :half], g).transpose(-3, -2).flatten(-2)), v
    x = rec.view(torch.float16).float()
    k = x[..., :64 * d].reshape(*lead, 4, d // 32, 4, 16, 8).permute(*range(n0), n0, n0 + 3, n0 + 1, n0 + 2, n0 + 4)
    v = x[..., 64 * d:].reshape(*lead, d // 16, 2, 4, 16, 8).permute(*range(n0), n0 + 2, n0 + 1, n0 + 4, n0, n0 + 3)
    return _key_order(k.reshape(*lead, 64, d)), v.reshape(*lead, 64, d)


# ---------------------------------------------------------------------------
# Inputs.
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _ints(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _cu(counts, dev):
    return _ints([0] + [int(x) for x in np.cumsum(counts)], dev)


def _dealt(pages, gen, dev):
    """Table [batch, most] of sequences whose pages are spread over a pool of one page more; -1 behind their ends."""
    total, most = sum(pages), max(pages)
    free = torch.randperm(total + 1, generator=gen, device=dev).int()
    count = torch.tensor(pages, device=dev)
    column = torch.arange(most, device=dev)
    first = torch.cumsum(count, 0) - count
    return torch.where(column < count[:, None], free[(first[:, None] + column).clamp(max=total)], -1).contiguous()


def _scaling(c):
    """Arguments of the frequencies' stretch: trained for 8192 positions, parts between 1 and 32 turns over them."""
    if c["scale"] == "none":
        return {}
    out = {"scaling": c["scale"], "factor": c["factor"]}
    if c["scale"] == "parts":
        out.update(original_len=8192, low=1.0, high=32.0, magnitude=0.1 * math.log(c["factor"]) + 1.0)
    return out


def prepare(case, seed):
    c, dev = case, _device()
    gen = torch.Generator(device=dev).manual_seed(int(seed) & 0x7FFFFFFFFFFF)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    if c["kind"] == ROPE:
        t, hq, hkv, d = c["tokens"], c["hq"], c["hkv"], c["d"]
        qkv = normal(t, (hq + 2 * hkv) * d).half()
        # runs of neighbouring positions, as chunks of sequences have them
        start = torch.randint(0, max(1, c["far"] - min(t, 512)), (t // 512 + 1,), generator=gen, device=dev)
        at = torch.arange(t, device=dev)
        pos = (start[at // 512] + at % 512).clamp(max=c["far"] - 1).int()
        st = {"case": c, "qkv": qkv, "pos": pos, "q": qkv[:, :hq * d].unflatten(1, (hq, d)),
              "k": qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))}
        if own:
            import paper_2607_04302_amd as h4
            st["rope"] = h4.Rope(d, c["rot"], base=10000.0, interleaved=c["interleaved"], device=dev, **_scaling(c))
        return st
    lens, new, pages, old = _lengths(c), _new(c), _pages(c), _old_pages(c)
    b, total, most = c["batch"], sum(pages), max(pages)
    table = _dealt(pages, gen, dev)
    st = {"case": c, "table": table}
    if c["kind"] in (EXTEND, RELEASE):
        moved = total - sum(old)
        st["old"], st["to"] = _ints(old, dev), _ints(pages, dev)
        # a pool of which a quarter more is free than the call takes
        spare = moved // 4 + 7
        st["free"] = torch.cat([torch.randperm(moved + spare, generator=gen, device=dev).int() + total + 1])
        st["num_free"] = _ints([moved + spare if c["kind"] == EXTEND else spare], dev)
        st["out_free"] = torch.empty_like(st["num_free"])
        if c["kind"] == EXTEND:
            st["table"] = torch.where(torch.arange(most, device=dev) < st["old"][:, None], table, -1).contiguous()
            t = sum(new)
            st.update(lens=_ints([n - m for n, m in zip(lens, new)], dev), counts=_ints(new, dev), total=t, most=max(new),
                      out_lens=_ints([0] * b, dev), cu=_ints([0] * (b + 1), dev),
                      positions=torch.empty(t, dtype=torch.int32, device=dev),
                      slots=torch.empty(t, dtype=torch.int64, device=dev), shift=None)
            if c["evicted"]:
                st["shift"] = PAGE * torch.randint(0, 1000, (b,), generator=gen, device=dev).int()
        return st
    # the model's amplified key channels (x16) under Smooth-QK, and its scales: about their root
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    gain = np.ones((hkv, d), np.float32)
    s = None
    if c["smooth"]:
        g = np.random.default_rng(4242)
        for h in range(hkv):
            gain[h, g.choice(d, d // 32, replace=False)] = 16.0
        s = torch.from_numpy(np.sqrt(gain) * g.uniform(0.9, 1.1, (hkv, d)).astype(np.float32)).to(dev)
    gain = torch.from_numpy(gain).to(dev)
    pool = torch.empty((total + 1, hkv, _page_bytes(c) // hkv), dtype=torch.uint8, device=dev)
    for at in range(0, total + 1, 512):
        n = min(512, total + 1 - at)
        k, v = normal(n, hkv, PAGE, d) * gain[:, None], normal(n, hkv, PAGE, d).half()
        k = (k if s is None else k / s[:, None]).half()
        pool[at:at + n] = _page4(k.float(), v.float()) if c["fmt"] == "hif4" else _page16(k, v)
    st.update(s=s, pool=pool, lens=_ints(lens, dev), cu=_cu(new, dev), most=max(new), q=normal(sum(new), hq, d).half())
    if own:
        import paper_2607_04302_amd as h4
        st["cache"] = h4.PagedCache(pool, table, st["lens"], d, h4.OPERANDS_HIF4 if c["fmt"] == "hif4" else h4.OPERANDS_FP16)
    return st


# ---------------------------------------------------------------------------
# The plain forms.
def _plain_extend(c, x):
    lens, counts, table = x["lens"].long(), x["counts"].long(), x["table"].clone()
    have = (lens + PAGE - 1) // PAGE
    need = (lens + counts + PAGE - 1) // PAGE - have
    cu = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
    first = torch.cumsum(need, 0) - need
    column = torch.arange(table.shape[1], device=table.device)
    fresh = (column >= have[:, None]) & (column < (have + need)[:, None])
    which = x["num_free"].long() - 1 - (first[:, None] + column - have[:, None])
    table = torch.where(fresh, x["free"][which.clamp(0, x["free"].numel() - 1)], table)
    at = torch.arange(x["total"], device=table.device)
    row = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    place = lens[row] + at - cu[row]
    slots = table[row, place // PAGE].long() * PAGE + place % PAGE
    positions = place if x["shift"] is None else place + x["shift"][row]
    return {"table": table, "lens": (lens + counts).int(), "num_free": x["num_free"] - need.sum().int(), "cu": cu.int(),
            "positions": positions.int(), "slots": slots}


def _plain_release(c, x):
    first, to, table = x["old"].long(), x["to"].long(), x["table"]
    column = torch.arange(table.shape[1], device=table.device)
    gone = table[(column >= first[:, None]) & (column < to[:, None])]          # by rows
    free = x["free"].clone()
    at = x["num_free"].long() + torch.arange(gone.numel(), device=gone.device)
    free[at] = gone.flip(0)                                   # the first row's first page ends on top
    return {"free": free, "num_free": x["num_free"] + gone.numel()}


def _frequencies(c, dev):
    """Angles per position of the pairs, in 64 bits, and the factor of the rotated values."""
    r, f = c["rot"], c["factor"]
    i = torch.arange(r // 2, dtype=torch.float64, device=dev)
    base = 10000.0 * (f ** (r / (r - 2.0)) if c["scale"] == "ntk" else 1.0)
    w = base ** (-2.0 * i / r)
    if c["scale"] == "linear":
        w = w / f
    if c["scale"] == "parts":
        kept = ((8192 * w / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        w = w * (kept + (1.0 - kept) / f)
    return w, (0.1 * math.log(f) + 1.0 if c["scale"] == "parts" else 1.0)


def _plain_rope(c, x):
    w, magnitude = _frequencies(c, x["pos"].device)
    angle = x["pos"].double()[:, None] * w
    cos, sin = (magnitude * torch.cos(angle)).float()[:, None], (magnitude * torch.sin(angle)).float()[:, None]
    if c["transposed"]:
        sin = -sin
    r = c["rot"]

    def turned(y):
        y = y.float()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
        ta, tb = a * cos - b * sin, a * sin + b * cos
        t = torch.stack([ta, tb], -1).flatten(-2) if c["interleaved"] else torch.cat([ta, tb], -1)
        return torch.cat([t, y[..., r:]], -1).half()

    return {"q": turned(x["q"]), "k": turned(x["k"])}


def _plain_chunk(c, x):
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    group, dev, total = hq // hkv, x["q"].device, x["q"].shape[0]
    q = x["q"].view(total, hkv, group, d)
    q = (q if x["s"] is None else _round16(q.double() * x["s"].double()[:, None])).float()
    o = torch.zeros((total, hkv, group, d), device=dev)
    lse = torch.full((hkv, group, total), -math.inf, device=dev)
    at = 0
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        if not m:
            continue
        k, v = _page_values(c, x["pool"][x["table"][b, :(n + PAGE - 1) // PAGE].long()])
        k = k.transpose(0, 1).flatten(1, 2)[:, :n].transpose(1, 2).contiguous()        # [Hkv, D, n]
        v = v.transpose(0, 1).flatten(1, 2)[:, :n].contiguous()
        some = max(1, (1 << 28) // (hq * n))
        for i in range(0, m, some):
            j = min(m, i + some)
            rows = q[at + i:at + j].permute(1, 2, 0, 3).reshape(hkv, group * (j - i), d)
            s = torch.matmul(rows, k).view(hkv, group, j - i, n) / math.sqrt(d)
            seen = torch.arange(n, device=dev) <= n - m + torch.arange(i, j, device=dev)[:, None]
            s = torch.where(seen, s, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            l = p.sum(-1, keepdim=True)
            out = torch.matmul((p / l).view(hkv, group * (j - i), n), v)
            o[at + i:at + j] = out.view(hkv, group, j - i, d).permute(2, 0, 1, 3)
            lse[:, :, at + i:at + j] = (top + torch.log(l))[..., 0]
        at += m
    return {"o": o.view(total, hq, d).half(), "lse": lse.view(hq, total)}


def run(state):
    c, x = state["case"], state
    if not own:
        return {EXTEND: _plain_extend, RELEASE: _plain_release, ROPE: _plain_rope, CHUNK: _plain_chunk}[c["kind"]](c, x)
    import paper_2607_04302_amd as h4
    if c["kind"] == EXTEND:
        h4.hifa4_paged_extend(x["table"], x["lens"], x["counts"], x["free"], x["num_free"], x["total"], max_new=x["most"],
                              shift=x["shift"], out_lens=x["out_lens"], out_free=x["out_free"], cu_new=x["cu"],
                              positions=x["positions"], slots=x["slots"])
        return {"table": x["table"], "lens": x["out_lens"], "num_free": x["out_free"], "cu": x["cu"],
                "positions": x["positions"], "slots": x["slots"]}
    if c["kind"] == RELEASE:
        h4.hifa4_paged_release(x["table"], x["to"], x["free"], x["num_free"], first=x["old"], out_free=x["out_free"])
        return {"free": x["free"], "num_free": x["out_free"]}
    if c["kind"] == ROPE:
        q, k = h4.hifa4_rope(x["rope"], x["pos"], x["q"], x["k"], transposed=c["transposed"])
        return {"q": q, "k": k}
    o, lse = h4.hifa4_paged_chunk_fwd(x["cache"], x["q"], x["cu"], x["s"], max_new=x["most"])
    return {"o": o, "lse": lse}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions: every value looked up in the page's bytes by its own address.
def _addresses(d, dev):
    """Of each (key, channel) of a HIF4 record: byte and shift of the code, bytes of E2 and E3 and their bit, byte of the
    base; K, then V."""
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


def _exact_rope(c, x):
    """Each pair as a complex number times a unit one."""
    r, f = c["rot"], c["factor"]
    pos = x["pos"].cpu().numpy().astype(np.float64)
    w = np.array([(10000.0 * (f ** (r / (r - 2.0)) if c["scale"] == "ntk" else 1.0)) ** (-2.0 * i / r) for i in range(r // 2)])
    unit = 1.0
    if c["scale"] == "linear":
        w /= f
    if c["scale"] == "parts":
        share = np.clip((8192 * w / (2 * np.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        w = w * share + w / f * (1.0 - share)
        unit = 1.0 + 0.1 * math.log(f)
    by = unit * np.exp((-1j if c["transposed"] else 1j) * pos[:, None] * w)
    by = torch.from_numpy(by).to(x["pos"].device)[:, None]
    first = torch.arange(r // 2, device=by.device) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else r // 2)

    def turned(y):
        z = y.double()
        t = torch.complex(z[..., first], z[..., second]) * by
        z[..., first], z[..., second] = t.real, t.imag
        return z

    return {"q": turned(x["q"]), "k": turned(x["k"])}


def _exact_chunk(c, x):
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    group, total, dev = hq // hkv, x["q"].shape[0], x["q"].device
    o = torch.zeros((total, hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((hq, total), -math.inf, dtype=torch.float64, device=dev)
    at = 0
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        pages = x["table"][b, :(n + PAGE - 1) // PAGE].long()
        for h in range(hkv if m else 0):
            k, v = [a.flatten(0, 1)[:n] for a in _look_up(c, x["pool"][pages, h])]
            k = k.t().contiguous()
            q = x["q"][at:at + m, h * group:(h + 1) * group].double()
            if x["s"] is not None:
                q = q * x["s"][h].double()
                q = torch.from_numpy(q.cpu().numpy().astype(np.float16)).to(dev).double()
            some = max(1, (1 << 26) // n)
            for g in range(group):
                for i in range(0, m, some):
                    j = min(m, i + some)
                    s = torch.mm(q[i:j, g].contiguous(), k) / math.sqrt(d)
                    hidden = torch.arange(n, device=dev) > torch.arange(n - m + i, n - m + j, device=dev)[:, None]
                    s.masked_fill_(hidden, -math.inf)
                    z = torch.logsumexp(s, 1)
                    lse[h * group + g, at + i:at + j] = z
                    o[at + i:at + j, h * group + g] = torch.mm(torch.exp(s - z[:, None]), v)
        at += m
    return {"o": o, "lse": lse}


def _exact_extend(c, x):
    table, free = x["table"].cpu().numpy().copy(), list(x["free"].cpu().numpy()[:int(x["num_free"])])
    lens, cu, positions, slots = [], [0], [], []
    shift = x["shift"].cpu().numpy() if c["evicted"] else [0] * c["batch"]
    for b, (n, m) in enumerate(zip(_lengths(c), _new(c))):
        for j in range(_old_pages(c)[b], _pages(c)[b]):
            table[b, j] = free.pop()
        at = np.arange(n - m, n)
        positions.append(at + shift[b])
        slots.append(table[b, at // PAGE].astype(np.int64) * PAGE + at % PAGE)
        lens.append(n)
        cu.append(cu[-1] + m)
    return {"table": torch.from_numpy(table), "lens": _ints(lens, "cpu"), "num_free": _ints([len(free)], "cpu"),
            "cu": _ints(cu, "cpu"), "positions": torch.from_numpy(np.concatenate(positions).astype(np.int32)),
            "slots": torch.from_numpy(np.concatenate(slots))}


def _exact_release(c, x):
    table, free = x["table"].cpu().numpy(), x["free"].cpu().numpy().copy()
    n = int(x["num_free"])
    for b in reversed(range(c["batch"])):
        for j in reversed(range(_old_pages(c)[b], _pages(c)[b])):
            free[n] = table[b, j]
            n += 1
    return {"free": torch.from_numpy(free), "num_free": _ints([n], "cpu")}


def exact(case, seed):
    c = case
    x = prepare(c, seed)
    return {EXTEND: _exact_extend, RELEASE: _exact_release, ROPE: _exact_rope, CHUNK: _exact_chunk}[c["kind"]](c, x)
