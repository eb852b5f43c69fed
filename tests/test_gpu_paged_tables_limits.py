"""Page tables at sizes and counts where their index arithmetic ends, on the GPU, against tests/_paged_chunk.py."""
import numpy as np
import pytest

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
