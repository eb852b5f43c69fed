"""Rotary positions, page tables and the attention of new tokens: refusals before any GPU work, and the frequencies
(no GPU needed)."""
import ctypes
import os
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2607_04302_amd as h

FAKE = 1 << 12          # an aligned non-NULL address; never dereferenced (validation fails first)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(h.LIB_PATH):
        pytest.skip("libhifa4.so not built")
    return h.load_library()


def _turns(lib, rot=64, base=10000.0, scaling=0, factor=1.0, length=0.0, low=0.0, high=1.0):
    out = (ctypes.c_uint64 * 128)()
    status = lib.hifa4_rope_frequencies(rot, base, scaling, factor, length, low, high, out)
    return status if status else [int(x) for x in out[:rot // 2]]


PI = Fraction(3141592653589793238462643383279502884197, 10 ** 39)


@pytest.mark.parametrize("rot", [8, 24, 64, 256])
@pytest.mark.parametrize("base", [10000.0, 1e6, 1.5])
def test_frequencies(lib, rot, base):
    """Every frequency against w / (2 pi) 2^64, w from float64: off by its relative 2^-50, and by 2 for the last places."""
    i = np.arange(rot // 2)
    w0 = base ** (-2.0 * i / rot)
    parts = 4096 * w0 / (2 * np.pi)
    g = np.clip((parts - 1.0) / 31.0, 0, 1)
    ntk = (base * 4.0 ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
    for got, w in ((_turns(lib, rot, base), w0), (_turns(lib, rot, base, 1, 4.0), w0 / 4), (_turns(lib, rot, base, 2, 4.0), ntk),
                   (_turns(lib, rot, base, 3, 4.0, 4096.0, 1.0, 32.0), w0 * (g + (1 - g) / 4))):
        for x, y in zip(got, w):
            exact = Fraction(float(y)) / (2 * PI) * 2 ** 64
            assert abs(x - exact) <= exact / 2 ** 48 + 2


def test_frequencies_are_checked(lib):
    for rot in (0, -8, 12, 264):
        assert _turns(lib, rot=rot) == -2
    assert _turns(lib, scaling=4) == -1 and _turns(lib, scaling=-1) == -1
    for base in (1.0, 0.0, float("nan"), float("inf")):
        assert _turns(lib, base=base) == -1
    for factor in (0.5, float("nan"), float("inf")):
        assert _turns(lib, scaling=1, factor=factor) == -1
    for length, low, high in ((0.0, 1.0, 2.0), (9.0, 2.0, 2.0), (9.0, -1.0, 2.0), (9.0, 1.0, float("inf")), (float("nan"), 1.0, 2.0)):
        assert _turns(lib, scaling=3, factor=2.0, length=length, low=low, high=high) == -1
    assert lib.hifa4_rope_frequencies(64, 10000.0, 0, 1.0, 0.0, 0.0, 1.0, None) == -1
    for kw in (dict(scaling="other"), dict(rot_dim=12), dict(rot_dim=192), dict(rot_dim=0)):
        with pytest.raises(ValueError):
            h.Rope(128, device="cpu", **kw)
    with pytest.raises(ValueError):
        h.Rope(96, device="cpu")
    with pytest.raises(h.Hifa4Error):
        h.Rope(128, base=0.5, device="cpu")


def _rope(lib, d=128, rot=128, inter=0, trans=0, mag=1.0, turns=FAKE, tokens=4, pos=FAKE, hq=2, q=FAKE, qs=256, qo=FAKE, qos=256, hk=2,
          k=FAKE, ks=256, ko=FAKE, kos=256):
    return lib.hifa4_rope(d, rot, inter, trans, mag, turns, tokens, pos, hq, q, qs, qo, qos, hk, k, ks, ko, kos, None)


def test_rope_is_checked(lib):
    assert _rope(lib, d=96) == -2
    assert _rope(lib, rot=132) == -2 and _rope(lib, rot=136) == -2 and _rope(lib, rot=0) == -2
    assert _rope(lib, inter=2) == -1 and _rope(lib, trans=-1) == -1
    assert _rope(lib, mag=float("nan")) == -1
    assert _rope(lib, tokens=-1) == -1 and _rope(lib, tokens=1 << 25) == -2
    assert _rope(lib, hq=-1) == -1 and _rope(lib, hk=-1) == -1
    assert _rope(lib, hq=1 << 24, qs=1 << 31, qos=1 << 31) == -2
    for name in ("q", "qo", "k", "ko"):
        assert _rope(lib, **{name: None}) == -1
        assert _rope(lib, **{name: FAKE + 8}) == -1
    for name in ("qs", "qos", "ks", "kos"):
        assert _rope(lib, **{name: 248}) == -1 and _rope(lib, **{name: 260}) == -1 and _rope(lib, **{name: 0}) == -1
        assert _rope(lib, **{name: 1 << 31}) == -2
    assert _rope(lib, qos=264) == -1 and "in place" in h.hifa4_last_error()
    assert _rope(lib, turns=None) == -1 and _rope(lib, pos=None) == -1
    assert _rope(lib, turns=FAKE + 4) == -1 and _rope(lib, pos=FAKE + 2) == -1
    assert _rope(lib, tokens=0, q=None, k=None, turns=None) == 0 and _rope(lib, hq=0, hk=0, q=None, k=None) == 0
    with pytest.raises(ValueError):
        h.hifa4_rope(h.Rope(128, device="cpu"), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 128, dtype=torch.float16))


def _extend(lib, batch=2, mp=4, ptr=None, cap=8, total=4, new=4, **kw):
    p = dict(table=FAKE, lens=FAKE, counts=FAKE, free=FAKE, num=FAKE, shift=None, out_lens=FAKE, out_free=FAKE, cu=FAKE, pos=FAKE, slots=FAKE)
    p.update(kw)
    return lib.hifa4_paged_extend(batch, mp, p["table"], p["lens"], p["counts"], p["free"], cap, p["num"], p["shift"], total, new,
                                  p["out_lens"], p["out_free"], p["cu"], p["pos"], p["slots"], None)


def test_extend_is_checked(lib):
    assert _extend(lib, batch=0) == -1 and _extend(lib, mp=0) == -1 and _extend(lib, cap=0) == -1
    assert _extend(lib, mp=1 << 25) == -2 and _extend(lib, batch=1 << 22) == -2 and _extend(lib, batch=1 << 15, mp=1 << 15) == -2
    assert _extend(lib, total=-1) == -1 and _extend(lib, new=-1) == -1
    for name in ("table", "lens", "counts", "free", "num", "out_lens", "out_free", "cu", "pos", "slots"):
        assert _extend(lib, **{name: None}) == -1
        assert _extend(lib, **{name: FAKE + 2}) == -1
    assert _extend(lib, shift=FAKE + 2) == -1 and _extend(lib, slots=FAKE + 4) == -1
    assert _extend(lib, batch=1 << 14, mp=1 << 15, total=2 ** 31 - 1, new=1 << 22) == -2


def _release(lib, batch=2, mp=4, cap=8, nbytes=12, **kw):
    p = dict(table=FAKE, first=None, to=FAKE, free=FAKE, num=FAKE, out=FAKE, ws=FAKE)
    p.update(kw)
    return lib.hifa4_paged_release(batch, mp, p["table"], p["first"], p["to"], p["free"], cap, p["num"], p["out"], p["ws"], nbytes, None)


def test_release_is_checked(lib):
    assert _release(lib, batch=0) == -1 and _release(lib, mp=0) == -1 and _release(lib, cap=-1) == -1
    assert _release(lib, mp=1 << 25) == -2
    for name in ("table", "to", "free", "num", "out"):
        assert _release(lib, **{name: None}) == -1
        assert _release(lib, **{name: FAKE + 2}) == -1
    assert _release(lib, first=FAKE + 1) == -1 and _release(lib, ws=FAKE + 2) == -1
    assert _release(lib, ws=None) == -3 and _release(lib, nbytes=11) == -3
    assert lib.hifa4_paged_release_workspace_bytes(2) == 12 and lib.hifa4_paged_release_workspace_bytes(0) == 0


def _chunk(lib, c=None, hq=4, total=6, new=3, cu=FAKE, q=FAKE, s=None, o=FAKE, lse=FAKE, ws=FAKE, nbytes=1 << 40, **kw):
    base = dict(batch=2, num_heads_kv=2, head_dim=128, operands=0, num_pages=8, max_pages=4, pool=FAKE, block_table=FAKE, seq_lens=FAKE,
                v_tail=None)
    base.update(kw)
    c = h.PagedCacheDesc(**base)
    need = lib.hifa4_paged_chunk_workspace_bytes(ctypes.byref(c), hq, total, new)
    return lib.hifa4_paged_chunk_fwd(ctypes.byref(c), hq, total, new, cu, q, s, o, lse, ws, need - 1 if nbytes is None else nbytes, None)


def test_chunk_is_checked(lib):
    assert _chunk(lib, head_dim=96) == -2 and _chunk(lib, num_heads_kv=0) == -1 and _chunk(lib, operands=2) == -1
    assert _chunk(lib, batch=0) == -1 and _chunk(lib, max_pages=1 << 25) == -2
    for name in ("pool", "block_table", "seq_lens"):
        assert _chunk(lib, **{name: None}) == -1
    assert _chunk(lib, hq=0) == -1 and _chunk(lib, hq=3) == -2
    assert _chunk(lib, total=-1) == -1 and _chunk(lib, new=-1) == -1
    assert _chunk(lib, total=1 << 29, new=1) == -2
    assert _chunk(lib, batch=1 << 20, total=1 << 24, new=1 << 20, num_heads_kv=64, hq=64) == -2
    for name in ("cu", "q", "o", "lse"):
        assert _chunk(lib, **{name: None}) == -1
        assert _chunk(lib, **{name: FAKE + 2}) == -1
    assert _chunk(lib, s=FAKE + 8) == -1 and _chunk(lib, ws=FAKE + 8) == -1
    assert _chunk(lib, ws=None) == -3 and _chunk(lib, nbytes=None) == -3
    assert _chunk(lib, total=0) == 0 and _chunk(lib, new=0) == 0
    assert lib.hifa4_paged_chunk_workspace_bytes(None, 4, 6, 3) == 0
