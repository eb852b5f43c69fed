"""The chunk attention, page table and rotation kernels as compiled: the copies into
LDS alone write M0, each immediately before its copy; inline statements keep the
waits of matrix instructions; no register is spilled or fetched from scratch among
them (which would wait for every copy under way); no packed fp32 instruction."""
import re

import pytest

from _asm import compile_to_asm
from test_asm_mfma_waits import _faults
from test_m0_guard import _hipcc

pytestmark = pytest.mark.skipif(_hipcc() is None, reason="hipcc not available")


def _code(text):
    lines = [l.split(";")[0].strip() for l in text.splitlines()]
    return [l for l in lines if l and not l.startswith((".", "_", "#")) and not l.endswith(":")]


def _m0_faults(code):
    found, copies = [], 0
    for i, l in enumerate(code):
        if re.search(r"\bm0\b", l):
            nxt = code[i + 1] if i + 1 < len(code) else ""
            if not l.startswith("s_mov_b32 m0,") or not nxt.startswith("global_load_lds_dwordx4") or ", s[" not in nxt:
                found.append((l, nxt))
            copies += 1
        elif l.startswith("global_load_lds") and not code[i - 1].startswith("s_mov_b32 m0,"):
            found.append((code[i - 1], l))
    return found, copies


def _scratch_in_products(text):
    """Blocks with more than eight matrix instructions, or a copy into LDS, that touch scratch memory."""
    found, blocks = [], 0
    for block in re.split(r"(?m)^(?=\S+:)", text):
        ops = [l.split(";")[0].strip() for l in block.splitlines()[1:]]
        if sum(o.startswith("v_mfma") for o in ops) > 8 or any(o.startswith("global_load_lds") for o in ops):
            blocks += 1
            if any(o.startswith("scratch_") for o in ops):
                found.append(block.splitlines()[0])
    return found, blocks


def test_compiled_chunk_kernels(tmp_path):
    text = compile_to_asm("hifa4_paged_chunk.hip", tmp_path)
    found, mfmas, inline = _faults(text)
    assert mfmas > 1000 and inline > 20 and not found
    found, copies = _m0_faults(_code(text))
    assert copies > 20 and not found, found[:3]
    found, blocks = _scratch_in_products(text)
    assert blocks > 20 and not found, found[:3]
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)


@pytest.mark.parametrize("source", ["hifa4_paged_tables.hip", "hifa4_rope.hip"])
def test_compiled_table_and_rotation_kernels(source, tmp_path):
    text = compile_to_asm(source, tmp_path)
    spills = re.findall(r"\.(?:vgpr|sgpr)_spill_count:\s+(\d+)", text)
    assert len(spills) >= 4 and not any(int(n) for n in spills)
    assert not re.search(r"\bm0\b|\bv_pk_(add|mul|fma)_f32\b", "\n".join(_code(text)))


@pytest.mark.parametrize("lines,bad", [
    (["s_mov_b32 m0, s4", "global_load_lds_dwordx4 v1, s[2:3]"], False),
    (["s_mov_b32 m0, s4", "s_nop 0", "global_load_lds_dwordx4 v1, s[2:3]"], True),
    (["s_mov_b32 s5, m0"], True),
    (["s_mov_b32 m0, s4", "global_load_lds_dwordx4 v1, s[2:3]", "global_load_lds_dwordx4 v1, s[2:3]"], True),
])
def test_the_check_of_m0_sees_planted_code(lines, bad):
    assert bool(_m0_faults(lines)[0]) == bad


def test_the_check_of_scratch_sees_planted_code():
    block = ["A:"] + ["\tv_mfma_x v[0:3], v[4:7], v[8:11], 0"] * 9
    assert _scratch_in_products("\n".join(block))== ([], 1)
    assert _scratch_in_products("\n".join(block + ["\tscratch_load_dword v1, off, off"])) == (["A:"], 1)
