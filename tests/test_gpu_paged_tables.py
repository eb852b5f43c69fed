"""Pages dealt out and put back on the GPU, against tests/_paged_chunk.py."""
import numpy as np
import pytest
import torch

import _paged_chunk as C
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np

pytestmark = pytest.mark.gpu


def _state(rng, lens, mp, spare):
    pages = [-(-max(0, min(n, 64 * mp)) // 64) for n in lens]
    order = rng.permutation(sum(pages) + spare).astype(np.int32)
    table = np.full((len(lens), mp), -7, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    free = np.concatenate([order[at:], np.full(5, -9, np.int32)])
    return table, free, spare


def _extend(table, lens, counts, free, num, max_total, max_new=None, shift=None, in_place=False):
    t, l, f, n = to_gpu(table), to_gpu(np.asarray(lens, np.int32)), to_gpu(free), to_gpu(np.array([num], np.int32))
    out = {} if in_place else {"out_lens": torch.full_like(l, -5), "out_free": torch.full_like(n, -5)}
    cu, pos, slots = h.hifa4_paged_extend(t, l, to_gpu(np.asarray(counts, np.int32)), f, n, max_total, max_new=max_new,
                                          shift=None if shift is None else to_gpu(np.asarray(shift, np.int32)), **out)
    want = C.extend(table, lens, counts, free, num, max_total, max_total if max_new is None else max_new, shift)
    got = (t, out.get("out_lens", l), out.get("out_free", n), cu, pos, slots)
    for x, y, name in zip(got, want, ("table", "lens", "free", "cu", "positions", "slots")):
        assert np.array_equal(to_np(x).reshape(-1), np.asarray(y).reshape(-1)), name
    assert np.array_equal(to_np(f), free)
    if not in_place:
        assert np.array_equal(to_np(l), lens) and int(n) == num
    return t, got


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("most", [1, 3, 130, 4000])
def test_extend_random(seed, most, in_place):
    rng = np.random.default_rng(seed + most)
    batch = (1, 7, 70, 1500)[seed]
    mp = 70
    lens = [int(x) for x in rng.integers(0, 400, batch)]
    counts = [int(x) for x in rng.integers(0, most + 1, batch)]
    table, free, num = _state(rng, lens, mp, sum(counts) // 64 + batch + 3)
    _extend(table, lens, counts, free, num, sum(counts) + (seed * 37) % 50, shift=rng.integers(0, 1000, batch) if seed % 2 else None,
            in_place=in_place)


@pytest.mark.parametrize("much", [1, 5000])
def test_extend_refuses_rows_in_order(much):
    """Rows that need more pages than are left, more tokens than max_total, more than their table or max_new."""
    rng = np.random.default_rng(1)
    lens = [64, 10, 63, 0, 100, 64 * 80, 64 * 80 - 1, 20]
    counts = [much, 3, 2, 64 * much // 5000 + 1, 28, 1, 1, 7]
    for spare in (0, 1, 2, 3, 40, 200):
        for cut in (0, 1, 2, 3, 10):
            table, free, num = _state(rng, lens, 80, spare)
            _extend(table, lens, counts, free, num, max(0, sum(counts) - cut * 9))
            _extend(table, lens, counts, free, num, sum(counts), max_new=27)


@pytest.mark.parametrize("tokens", [4096, 4097, 20000])
def test_extend_counts_and_lengths_outside_the_contract(tokens):
    rng = np.random.default_rng(2)
    lens = [-3, 64 * 400 + 9, 5, 0, 77]
    counts = [4, 3, -1, tokens - 40, -2 ** 31]
    table, free, num = _state(rng, lens, 400, 900)
    _extend(table, lens, counts, free, num, tokens)
    _extend(table, lens, [2 ** 31 - 1] * 5, free, num, tokens)
    _extend(table, lens, counts, free, len(free) + 100, tokens)      # (the stack holds no more than its buffer)
    _extend(table, lens, counts, free, -4, tokens)
    table[4, 1] = -1                                                  # a page that is none
    _extend(table, lens, [0, 0, 0, 0, 60], free, num, tokens)
    _extend(table, lens, [0] * 5, free, num, 0)


def test_extend_of_a_large_batch():
    """More rows than one pass over the batch takes, and more pages of one row than one workgroup fills."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 130, 2500)]
    counts = [int(x) for x in rng.integers(0, 4, 2500)]
    table, free, num = _state(rng, lens, 4, 3000)
    _extend(table, lens, counts, free, num, sum(counts))
    lens, counts = [100, 64 * 3000, 0], [64 * 2000 + 3, 130, 30000]
    table, free, num = _state(rng, lens, 4000, 2600)
    _extend(table, lens, counts, free, num, sum(counts))


@pytest.mark.parametrize("seed", range(6))
def test_release(seed):
    rng = np.random.default_rng(seed)
    batch, mp = (1, 9, 300, 4, 65, 2)[seed], (1, 40, 7, 3000, 64, 700)[seed]
    table = rng.permutation(batch * mp).astype(np.int32).reshape(batch, mp)
    table[rng.random(table.shape) < 0.1 * (seed % 3)] = -1
    first = rng.integers(-2, mp + 2, batch).astype(np.int32) if seed % 2 else None
    to = rng.integers(-3, mp + 9, batch).astype(np.int32)
    for num, room in ((0, batch * mp), (17, batch * mp + 17), (5, 5 + batch * mp // 3), (30, 30), (-1, batch * mp), (40, 31)):
        free = rng.integers(10 ** 6, 2 * 10 ** 6, room).astype(np.int32)
        want, n = C.release(table, to, free, num, first)
        t, f, c = to_gpu(table), to_gpu(free), to_gpu(np.array([num], np.int32))
        out = h.hifa4_paged_release(t, to_gpu(to), f, c, first=None if first is None else to_gpu(first))
        assert out is c and int(c) == n
        assert np.array_equal(to_np(f), want) and np.array_equal(to_np(t), table)
        c2 = to_gpu(np.array([num], np.int32))
        f2 = to_gpu(free)
        o2 = h.hifa4_paged_release(t, to_gpu(to), f2, c2, first=None if first is None else to_gpu(first), out_free=torch.empty_like(c2),
                                   workspace=h.Workspace())
        assert int(o2) == n and int(c2) == num and torch.equal(f, f2)


@pytest.mark.parametrize("batch,mp", [(64, 64), (1, 4096), (4096, 1), (1, 4097), (17, 241)])
def test_release_where_one_launch_ends(batch, mp):
    """4096 places and one more; every second entry is none."""
    rng = np.random.default_rng(batch)
    table = rng.permutation(batch * mp).astype(np.int32).reshape(batch, mp)
    table.reshape(-1)[::2] *= -1
    free = rng.integers(10 ** 6, 2 * 10 ** 6, batch * mp + 3).astype(np.int32)
    want, n = C.release(table, np.full(batch, mp, np.int32), free, 3)
    f, c = to_gpu(free), to_gpu(np.array([3], np.int32))
    h.hifa4_paged_release(to_gpu(table), to_gpu(np.full(batch, mp, np.int32)), f, c)
    assert int(c) == n and np.array_equal(to_np(f), want)


def test_release_undoes_extend():
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 300, 40)]
    counts = [int(x) for x in rng.integers(0, 700, 40)]
    table, free, num = _state(rng, lens, 20, 500)
    t, (_, new_lens, left, *_rest) = _extend(table, lens, counts, free, num, sum(counts))
    f = to_gpu(free)
    f[int(left):] = -1
    had, has = to_gpu(np.array([-(-n // 64) for n in lens], np.int32)), ((new_lens + 63) // 64).int()
    h.hifa4_paged_release(t, has, f, left, first=had)
    assert int(left) == num and np.array_equal(to_np(f)[:num], free[:num])


def test_evicted_pages_go_back():
    rng = np.random.default_rng(6)
    lens = [64 * 9, 30, 64 * 5 + 1]
    table, free, num = _state(rng, lens, 12, 4)
    free = np.concatenate([free[:4], np.zeros(30, np.int32)])
    t, l, f, c = to_gpu(table), to_gpu(np.array(lens, np.int32)), to_gpu(free), to_gpu(np.array([num], np.int32))
    w = to_gpu(rng.random(table.shape).astype(np.float32))
    freed, n = h.hifa4_paged_evict(t, l, w, budget=4, first=1, last=1)
    h.hifa4_paged_release(freed, n, f, c)
    gone = to_np(freed)
    want = [x for b in range(3) for x in gone[b] if x >= 0]
    assert len(want) == 5 + 2 and int(c) == num + 7
    assert list(to_np(f)[num:num + 7]) == want[::-1]


def test_tables_captured():
    """Extend and release in one graph, replayed with other lengths, counts and stacks."""
    rng = np.random.default_rng(7)
    batch, mp = 33, 60
    t, l = torch.zeros((batch, mp), dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    counts, free = torch.zeros_like(l), torch.zeros(3000, dtype=torch.int32, device="cuda")
    num, first, to = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros_like(l), torch.zeros_like(l)
    out_free = torch.zeros_like(num)
    for max_total in (900, 9000):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                cu, pos, slots = h.hifa4_paged_extend(t, l, counts, free, num, max_total, shift=first)
                h.hifa4_paged_release(t, to, free, num, first=first, out_free=out_free)
        torch.cuda.synchronize()
        for _ in range(4):
            lens = [int(x) for x in rng.integers(0, 300, batch)]
            cnt = [int(x) for x in rng.integers(0, max_total // 20, batch)]
            table, stack, n = _state(rng, lens, mp, int(rng.integers(1, 400)))
            table[table < 0] = -1
            some = rng.integers(0, 3, batch).astype(np.int32)
            pad = np.concatenate([stack, np.zeros(3000 - len(stack), np.int32)])
            for x, y in ((t, table), (l, lens), (counts, cnt), (free, pad), (num, [n]), (first, some), (to, [3] * batch)):
                x.copy_(torch.from_numpy(np.asarray(y, np.int32)))
            want = C.extend(table, lens, cnt, pad, n, max_total, max_total, some)
            left, back = C.release(want[0], [3] * batch, pad, want[2], some)
            graph.replay()
            torch.cuda.synchronize()
            for x, y in ((t, want[0]), (l, want[1]), (num, [want[2]]), (cu, want[3]), (pos, want[4]), (slots, want[5]),
                         (free, left), (out_free, [back])):
                assert np.array_equal(to_np(x).reshape(-1), np.asarray(y).reshape(-1))
            torch.zeros(100, device="cuda").sum()


def test_tables_on_other_streams():
    """Two threads' calls on streams of their own."""
    rng = np.random.default_rng(8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    cases = []
    for s in streams:
        lens = [int(x) for x in rng.integers(0, 300, 50)]
        table, free, num = _state(rng, lens, 60, 900)
        cases.append((table, free, num, lens))
    done = []
    for s, (table, free, num, lens) in zip(streams, cases):
        with torch.cuda.stream(s):
            t, f, c = to_gpu(table), to_gpu(free), to_gpu(np.array([num - 100], np.int32))
            to = to_gpu(np.array([-(-n // 64) for n in lens], np.int32))
            s.synchronize()
            for _ in range(20):
                c.fill_(num - 100)
                h.hifa4_paged_release(t, to, f, c)
            done.append((f, c, to))
    torch.cuda.synchronize()
    for (f, c, to), (table, free, num, lens) in zip(done, cases):
        want, n = C.release(table, to_np(to), free, num - 100)
        assert int(c) == n and np.array_equal(to_np(f), want)
