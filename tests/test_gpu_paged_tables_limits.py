"""Page tables at sizes and counts where their index arithmetic ends, on the GPU, against tests/_paged_chunk.py."""
import threading

import numpy as np
import pytest
import torch

import _paged_chunk as C
import paper_2607_04302_amd as h
from _gpu_util import to_gpu, to_np
from test_gpu_paged_tables import _extend, _state

pytestmark = pytest.mark.gpu


def test_extend_of_more_workgroups_than_31_bits_of_threads():
    """1025 rows and max_total 2^24 + 8192, max_new by default: 8400900 workgroups of 256 threads."""
    rng = np.random.default_rng(9)
    lens = [int(x) for x in rng.integers(0, 130, 1025)]
    counts = [int(x) for x in rng.integers(0, 8, 1025)]
    table, free, num = _state(rng, lens, 4, 2000)
    total = (1 << 24) + 8192
    assert 1025 * -(-total // 2048) * 256 > 1 << 31
    _extend(table, lens, counts, free, num, total)


@pytest.mark.parametrize("batch,max_total,max_new", [(1025, 0, None), (1025, 0, 7), (5, 5000, 0), (1025, 10, 0), (1025, 5000, 0),
                                                     (1024, 0, None), (1024, 10, 0)])
def test_extend_of_no_tokens(batch, max_total, max_new):
    """An idle step: no row may get a token; lengths and stack stay, every position and slot is -1."""
    rng = np.random.default_rng(10)
    lens = [int(x) for x in rng.integers(0, 130, batch)]
    counts = [int(x) for x in rng.integers(0, 8, batch)]
    table, free, num = _state(rng, lens, 4, 100)
    _, (_, new_lens, left, cu, pos, slots) = _extend(table, lens, counts, free, num, max_total, max_new)
    assert int(cu.abs().max()) == 0 and int(left) == num and new_lens.tolist() == lens
    assert bool((pos == -1).all()) and bool((slots == -1).all())


@pytest.mark.parametrize("batch,mp", [(3, 40), (3, 3000)])
def test_release_cuts_places_to_the_row(batch, mp):
    """First and last places up to the ends of 32 bits, in one launch and in two."""
    rng = np.random.default_rng(11)
    table = rng.permutation(batch * mp).astype(np.int32).reshape(batch, mp)
    ends = [-2 ** 31, -1, 0, mp - 1, mp, 2 ** 31 - 256, 2 ** 31 - 255, 2 ** 31 - 1]
    for first in ends:
        for to in ends:
            firsts, tos = np.array([0, first, mp // 2], np.int32), np.array([mp // 3, to, mp], np.int32)
            free = rng.integers(10 ** 6, 2 * 10 ** 6, batch * mp + 3).astype(np.int32)
            want, n = C.release(table, tos, free, 3, firsts)
            f, c = to_gpu(free), to_gpu(np.array([3], np.int32))
            h.hifa4_paged_release(to_gpu(table), to_gpu(tos), f, c, first=to_gpu(firsts))
            assert int(c) == n and np.array_equal(to_np(f), want), (first, to)


def test_tables_of_two_threads():
    """Two threads release and extend at the same time, each on a stream of its own, with the workspaces of calls that
    bring none; more than 4096 places, so that a release passes counts from one kernel to the next."""
    rng = np.random.default_rng(13)
    cases, got = [], [None, None]
    for i in range(2):
        lens = [int(x) for x in rng.integers(0, 300, 50 + i)]
        table, free, num = _state(rng, lens, 120, 900)
        counts = [int(x) for x in rng.integers(0, 90, len(lens))]
        cases.append((table, free, num, lens, counts))
    ready = threading.Barrier(2)

    def work(i):
        table, free, num, lens, counts = cases[i]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            t, f, n = to_gpu(table), to_gpu(free), to_gpu(np.array([num], np.int32))
            l, c = to_gpu(np.array(lens, np.int32)), to_gpu(np.array(counts, np.int32))
            had = to_gpu(np.array([-(-x // 64) for x in lens], np.int32))
            stream.synchronize()
            ready.wait(60)
            for _ in range(40):
                cu, pos, slots = h.hifa4_paged_extend(t, l, c, f, n, 9000, out_lens=torch.empty_like(l), out_free=(left := torch.empty_like(n)))
                has = (l + (cu[1:] - cu[:-1]) + 63) // 64
                h.hifa4_paged_release(t, has.int(), f, left, first=had)
            stream.synchronize()
            got[i] = [to_np(x) for x in (t, f, left, cu, pos, slots)]

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for x in threads:
        x.start()
    for x in threads:
        x.join(100)
    for (table, free, num, lens, counts), x in zip(cases, got):
        t, _, _, cu, pos, slots = C.extend(table, lens, counts, free, num, 9000, 9000)
        assert np.array_equal(x[0], t) and np.array_equal(x[1], free) and int(x[2][0]) == num
        assert np.array_equal(x[3], cu) and np.array_equal(x[4], pos) and np.array_equal(x[5], slots)
