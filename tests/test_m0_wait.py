"""The copies into LDS take their LDS address from M0.  The instruction set asks for one wait state between a scalar
write of M0 and such a copy, and the hardware does not insert it: in the machine code of the kernels (this library's
sources, compiled and listed here) no copy follows its write of M0 directly."""
import os
import re
import shutil
import subprocess

import pytest

from test_m0_guard import ROOT, _hipcc


def _objdump():
    for cand in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")):
        if cand and os.path.exists(cand):
            return cand
    return None


def _machine_code(source, folder):
    out = os.path.join(str(folder), source + ".o")
    subprocess.run([_hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "--no-gpu-bundle-output", "-c",
                    "-x", "hip", os.path.join(ROOT, "paper_2607_04302_amd", "csrc", source), "-o", out],
                   check=True, capture_output=True, timeout=600)
    text = subprocess.run([_objdump(), "-d", "--mcpu=gfx950", out], check=True, capture_output=True, timeout=600).stdout.decode()
    return [l.split("//")[0].strip() for l in text.splitlines() if l.startswith("\t")]


def _copies_without_wait(code):
    """(copies into LDS, those that directly follow a write of M0)"""
    copies = [i for i, l in enumerate(code) if re.match(r"(global|scratch)_load_lds_|buffer_load_.*\blds\b", l)]
    return len(copies), [code[i - 1:i + 1] for i in copies if i and re.match(r"s_\w+ m0,", code[i - 1])]


@pytest.mark.skipif(_hipcc() is None or _objdump() is None, reason="hipcc or llvm-objdump not available")
@pytest.mark.parametrize("source", ["hifa4_attn.hip", "hifa4_decode.hip", "hifa4_paged_chunk.hip"])
def test_copies_into_lds_wait_for_m0(source, tmp_path):
    copies, found = _copies_without_wait(_machine_code(source, tmp_path))
    assert copies > 10 and not found, (len(found), found[:3])


@pytest.mark.parametrize("between,bad", [([], 1), (["s_nop 0"], 0), (["v_add_u32_e32 v1, 0x400, v1"], 0)])
def test_the_check_sees_planted_code(between, bad):
    code = ["s_mov_b32 m0, s4"] + between + ["global_load_lds_dwordx4 v1, s[2:3]"]
    assert _copies_without_wait(code) == (1, [["s_mov_b32 m0, s4", code[-1]]] * bad)
