"""Index arithmetic of the page tables' kernels at the largest sizes that the entry points accept (no GPU needed)."""
import ctypes

import pytest

from _host import compile_host, have_compiler

SOURCE = """
#include "hifa4_paged_tables.h"
extern "C" {
int64_t tail_first(int total, uint32_t block, int thread) { return hifa4::tail_first(total, block, thread); }
int64_t tail_step(uint32_t blocks) { return hifa4::tail_step(blocks); }
int fill_end(int n, int i0) { return hifa4::fill_end(n, i0); }
int extend_chunks(int max_new) { return hifa4::extend_chunks(max_new); }
int release_first(int first, int max_pages) { return hifa4::release_first(first, max_pages); }
int release_end(int to, int max_pages) { return hifa4::release_end(to, max_pages); }
int fill_threads() { return hifa4::kFillThreads; }
int fill_tokens() { return hifa4::kFillTokens; }
}
"""


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    if not have_compiler():
        pytest.skip("g++ not available")
    lib = compile_host(SOURCE, tmp_path_factory.mktemp("tables"))
    lib.tail_first.restype, lib.tail_first.argtypes = ctypes.c_int64, [ctypes.c_int, ctypes.c_uint32, ctypes.c_int]
    lib.tail_step.restype, lib.tail_step.argtypes = ctypes.c_int64, [ctypes.c_uint32]
    return lib


@pytest.mark.parametrize("total", [0, 256, 4097, 1 << 24, 2 ** 31 - 1])
@pytest.mark.parametrize("blocks", [1, 1025, (1 << 23) - 1, 1 << 23, 8400900, (1 << 24) - 1])
def test_every_entry_of_the_tail_has_one_thread(index, blocks, total):
    """The threads of a launch begin at total, total + 1, ... without a gap and step over all of them: none
    begins before the tail, each entry has one thread, and every thread passes any max_total."""
    threads = index.fill_threads()
    step = index.tail_step(blocks)
    assert step == blocks * threads
    for block in sorted({0, 1, blocks // 2, blocks - 1} & set(range(blocks))):
        for thread in (0, threads - 1):
            assert index.tail_first(total, block, thread) == total + block * threads + thread
    assert index.tail_first(total, blocks - 1, threads - 1) + 1 == total + step


@pytest.mark.parametrize("n", [1, 2047, 2048, 2049, 2 ** 31 - 2048, 2 ** 31 - 2047, 2 ** 31 - 64])
def test_the_parts_of_a_row_end_where_the_next_begin(index, n):
    part = index.fill_tokens()
    last = (n - 1) // part * part
    assert index.fill_end(n, last) == n
    for i0 in {0, last // 2 // part * part, last - part} & set(range(0, last, part)):
        assert index.fill_end(n, i0) == i0 + part


@pytest.mark.parametrize("max_new", [0, 1, 2047, 2048, 2049, 2 ** 31 - 1])
def test_every_row_has_a_workgroup(index, max_new):
    assert index.extend_chunks(max_new) == max(1, -(-max_new // index.fill_tokens()))


@pytest.mark.parametrize("max_pages", [1, 64, 5000, (1 << 25) - 1])
def test_released_places_are_cut_to_the_row(index, max_pages):
    for x in (-2 ** 31, -1, 0, 1, max_pages - 1, max_pages, max_pages + 1, 2 ** 31 - 256, 2 ** 31 - 1):
        assert index.release_first(x, max_pages) == min(max(x, 0), max_pages)
        assert index.release_end(x, max_pages) == min(x, max_pages)
