"""Rotary positions of tensors whose strides say nothing, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2607_04302_amd as h
from _gpu_util import to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [0, 1])
@pytest.mark.parametrize("width", [1001, 1024, 100000])
def test_one_token_of_any_row_length(tokens, width):
    """One token's row of a buffer whose rows are no multiple of 8 elements apart, new and in place (also by a view
    of the same memory with another stride), as a contiguous copy is rotated."""
    rng = np.random.default_rng(width)
    rope = h.Rope(128, base=1e6)
    pos = to_gpu(np.full(tokens, 12345, np.int32))
    rows = to_gpu(rng.standard_normal((2, width)).astype(np.float16))
    q = torch.as_strided(rows, (tokens, 3, 128), (width, 128, 1), 16)
    k = torch.as_strided(rows, (tokens, 1, 128), (width, 128, 1), 400)
    assert q.stride(0) == width
    want_q, want_k = h.hifa4_rope(rope, pos, q.contiguous(), k.contiguous())
    got_q, got_k = h.hifa4_rope(rope, pos, q, k)
    assert torch.equal(got_q, want_q) and torch.equal(got_k, want_k)
    before = rows.clone()
    same = torch.as_strided(rows, q.shape, (2048, 128, 1), 16)
    h.hifa4_rope(rope, pos, q, None, q_out=same)
    before[:tokens, 16:16 + 3 * 128] = want_q.flatten(1)
    assert torch.equal(rows, before)
