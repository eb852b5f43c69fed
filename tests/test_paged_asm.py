"""The paged decode kernels as compiled: no inline instruction stands beside
their matrix instructions (so every wait between the two is the compiler's),
no scalar or vector register is spilled, and no packed fp32 instruction is in them."""
import re

import pytest

from _asm import compile_to_asm
from test_asm_mfma_waits import _faults
from test_m0_guard import _hipcc


@pytest.mark.skipif(_hipcc() is None, reason="hipcc not available")
@pytest.mark.parametrize("source", ["hifa4_paged_decode.hip", "hifa4_paged.hip"])
def test_compiled_paged_kernels(source, tmp_path):
    text = compile_to_asm(source, tmp_path)
    found, mfmas, inline = _faults(text)
    assert not found
    if source == "hifa4_paged_decode.hip":
        assert mfmas > 100 and inline == 0
    else:
        assert mfmas == 0
    spills = re.findall(r"\.(?:vgpr|sgpr)_spill_count:\s+(\d+)", text)
    assert len(spills) >= 12 and not any(int(n) for n in spills)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
