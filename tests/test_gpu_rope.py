"""Rotary positions on the GPU against float64."""
import math

import numpy as np
import pytest
import torch

import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np

pytestmark = pytest.mark.gpu

SCALINGS = {"none": {}, "linear": dict(factor=2.5), "ntk": dict(factor=4.0),
            "parts": dict(factor=8.0, original_len=4096, low=1.0, high=32.0, magnitude=1.25)}


def _frequencies(rot, scaling, base=10000.0, factor=1.0, original_len=0.0, low=0.0, high=1.0, magnitude=1.0):
    i = np.arange(rot // 2)
    if scaling == "ntk":
        base *= factor ** (rot / (rot - 2.0))
    w = base ** (-2.0 * i / rot)
    if scaling == "linear":
        w /= factor
    if scaling == "parts":
        g = np.clip((original_len * w / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        w = w * (g + (1 - g) / factor)
    return w


def _want(x, pos, rot, w, interleaved, magnitude, transposed):
    """Rotated x [T, H, D] and its bound.  The angle in float64 is off by 2^-52 of itself and so is the frequency; the
    kernel's cosine and sine by at most 2^-22 (angle cut at 2^-32 of a turn and rounded, 2^-23 in all; series and their
    roundings 2^-23), the products and their sum by three roundings of 2^-24, the result by 2^-11 or 2^-25."""
    x = x.astype(np.float64)
    angle = pos[:, None].astype(np.float64) * w
    c, s = magnitude * np.cos(angle)[:, None], magnitude * np.sin(angle)[:, None] * (-1 if transposed else 1)
    a = np.arange(rot // 2) * (2 if interleaved else 1)
    b = a + (1 if interleaved else rot // 2)
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    off = magnitude * (2.0 ** -22 + 4 * 2.0 ** -24 + 3 * 2.0 ** -52 * np.abs(angle))[:, None]
    bound = np.zeros_like(y)
    bound[..., a] = bound[..., b] = off * (np.abs(x[..., a]) + np.abs(x[..., b]))
    turned = bound > 0
    bound[turned] += (2.0 ** -11 * np.abs(y) + 2.0 ** -25)[turned]
    return y, bound


def _case(seed, tokens, hq, hk, d, rot, interleaved=False, scaling="none", far=40000, transposed=False, fused=False, in_place=False):
    rng = np.random.default_rng(seed)
    qkv = rng.standard_normal((tokens, hq + 2 * hk, d)).astype(np.float16)
    pos = rng.integers(0, far, tokens).astype(np.int32)
    kw = SCALINGS[scaling]
    rope = h.Rope(d, rot, interleaved=interleaved, scaling=scaling, **kw)
    t = to_gpu(qkv)
    q, k = t[:, :hq], t[:, hq:hq + hk]
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    oq, ok = h.hifa4_rope(rope, to_gpu(pos), q if hq else None, k if hk else None, transposed=transposed,
                          **({"q_out": q if hq else None, "k_out": k if hk else None} if in_place else {}))
    w = _frequencies(rot, scaling, **kw)
    for got, x in ((oq, qkv[:, :hq]), (ok, qkv[:, hq:hq + hk])):
        if x.shape[1] == 0:
            continue
        y, bound = _want(x, pos, rot, w, interleaved, kw.get("magnitude", 1.0), transposed)
        err = np.abs(to_np(got).astype(np.float64) - y)
        assert (err <= bound).all(), (err - bound).max()
    if fused:
        kept = to_np(t)[:, hq + hk if in_place else 0:]
        assert np.array_equal(kept, qkv[:, hq + hk if in_place else 0:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 8), (64, 24), (128, 128), (128, 64), (128, 40), (128, 120), (256, 256), (256, 64),
                                   (256, 248), (256, 16)])
def test_rope_layouts(d, rot, interleaved):
    _case(rot, 37, 6, 2, d, rot, interleaved)
    _case(rot, 5, 3, 1, d, rot, interleaved, transposed=True, fused=True, in_place=True)


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_scalings(scaling, interleaved):
    _case(1, 300, 4, 2, 128, 128, interleaved, scaling)
    _case(2, 300, 4, 2, 64, 32, interleaved, scaling, transposed=True)


@pytest.mark.parametrize("far", [1, 1 << 20, 1 << 27, 2 ** 31 - 1])
def test_rope_far_positions(far):
    _case(3, 200, 2, 2, 128, 128, far=far)
    _case(4, 200, 2, 2, 64, 48, True, "parts", far=far)


@pytest.mark.parametrize("tokens,hq,hk", [(1, 1, 0), (1, 0, 1), (1, 32, 8), (3, 71, 1), (4097, 8, 8), (5000, 32, 8), (0, 4, 2)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope_sizes(tokens, hq, hk, in_place):
    _case(5, tokens, hq, hk, 128, 128, fused=True, in_place=in_place)


def test_rope_is_exact_where_nothing_turns():
    rng = np.random.default_rng(6)
    x = to_gpu(rng.standard_normal((9, 3, 128)).astype(np.float16))
    out, _ = h.hifa4_rope(h.Rope(128), torch.zeros(9, dtype=torch.int32, device="cuda"), x)
    assert torch.equal(out, x)


def test_rope_leaves_rows_that_are_no_tokens():
    rng = np.random.default_rng(7)
    x = to_gpu(rng.standard_normal((50, 3, 64)).astype(np.float16))
    x[:, 1, 5] = math.nan
    pos = to_gpu(rng.integers(0, 99, 50).astype(np.int32))
    pos[::3] = -1
    pos[1] = -2 ** 31
    rope = h.Rope(64, 32)
    full, _ = h.hifa4_rope(rope, pos.clamp(min=0), x)
    out = torch.full_like(x, 7.0)
    got, none = h.hifa4_rope(rope, pos, x, q_out=out)
    assert none is None and got is out
    assert (out[pos < 0] == 7.0).all()
    assert torch.equal(out[pos >= 0].view(torch.int16), full[pos >= 0].view(torch.int16))
    bad = torch.isnan(full)
    assert bad[:, 1, [5, 21]].all() and int(bad.sum()) == 100        # a NaN reaches its pair and no other channel


def test_rope_transposed_is_the_gradient_and_the_inverse():
    """<R x, y> = <x, R' y>, and R' R x = x within the roundings of both; differences of R along single channels are
    the columns of R."""
    rng = np.random.default_rng(8)
    x, y = (to_gpu(rng.standard_normal((64, 4, 128)).astype(np.float16)) for _ in range(2))
    pos = to_gpu(rng.integers(0, 5000, 64).astype(np.int32))
    for kw in ({}, dict(interleaved=True, rot_dim=64)):
        rope = h.Rope(128, **kw)
        rx, _ = h.hifa4_rope(rope, pos, x)
        ry, _ = h.hifa4_rope(rope, pos, y, transposed=True)
        # every product is off by up to 2^-11 of its rounded factor, so a row's sum by that of its absolute terms (and
        # 2^-20 of both for cosine, sine and fp32)
        lhs, rhs = (rx.double() * y.double()).sum(-1), (x.double() * ry.double()).sum(-1)
        room = (2.0 ** -11 + 2.0 ** -19) * ((rx.double() * y.double()).abs().sum(-1) + (x.double() * ry.double()).abs().sum(-1))
        room += 2.0 ** -19 * (x.double().norm(dim=-1) * y.double().norm(dim=-1))
        assert ((lhs - rhs).abs() <= room).all()
        back, _ = h.hifa4_rope(rope, pos, rx, transposed=True)
        # two roundings of 2^-11 of values that are at most the pair's length
        r = rope.rot_dim
        pair = x.double()[..., :r].unflatten(-1, (r // 2, 2) if kw else (2, r // 2)).norm(dim=-1 if kw else -2)
        pair = pair.repeat_interleave(2, -1) if kw else torch.cat([pair, pair], -1)
        off = (back.double() - x.double()).abs()
        assert (off[..., :r] <= (2 ** 0.5 * 2.0 ** -11 + 2.0 ** -11 + 2.0 ** -18) * pair).all() and not off[..., r:].any()
        # a step of 1 in one channel: the difference is R's column, the gradient's row
        e = torch.zeros_like(x)
        e[:, :, 3] = 1.0
        column, _ = h.hifa4_rope(rope, pos, e)
        gy = (column.double() * y.double()).sum(-1)
        # the column's two values are rounded by 2^-11 of themselves (at most 1 each), the gradient by 2^-11 of itself
        tol = 2.0 ** -11 * ((column.double() * y.double()).abs().sum(-1) + ry[..., 3].double().abs()) + 2.0 ** -17 * y.double().abs().amax(-1)
        assert ((gy - ry[..., 3].double()).abs() <= tol).all()


def test_rope_captured_and_on_other_streams():
    rng = np.random.default_rng(9)
    x, k = (torch.zeros((40, n, 128), dtype=torch.float16, device="cuda") for n in (8, 2))
    pos = torch.zeros(40, dtype=torch.int32, device="cuda")
    rope = h.Rope(128, 96, interleaved=True)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            oq, ok = h.hifa4_rope(rope, pos, x, k)
    torch.cuda.synchronize()
    for _ in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape).astype(np.float16)))
        k.copy_(torch.from_numpy(rng.standard_normal(k.shape).astype(np.float16)))
        pos.copy_(torch.from_numpy(rng.integers(-3, 9999, 40).astype(np.int32)))
        there = pos >= 0
        graph.replay()
        torch.cuda.synchronize()
        eq, ek = h.hifa4_rope(rope, pos, x, k)
        assert torch.equal(eq[there], oq[there]) and torch.equal(ek[there], ok[there])
