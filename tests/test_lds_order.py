"""Data that the lanes of a wave hand one another through LDS.  The hardware
keeps a wave's LDS accesses in order; the compiler keeps an order only between
accesses of one lane that may meet, and knows nothing of the other lanes.  So in
the paged cache's kernels whose waves do so, compiled to LLVM IR, along every
path, a fence (that of a barrier, or one of the wave's own) lies between a store
to an LDS array and a load from it, and between a load and the next store."""
import os
import re
import subprocess

import pytest

from test_m0_guard import ROOT, _hipcc


def _ir(source, folder):
    out = os.path.join(str(folder), source + ".ll")
    cmd = [_hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S", "-emit-llvm", "-x", "hip",
           os.path.join(ROOT, "paper_2607_04302_amd", "csrc", source), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True, timeout=600)
    with open(out) as f:
        return f.read()


def _functions(text):
    for m in re.finditer(r"^define [^\n]*?@([\w.$]+)\([^\n]*\{\n(.*?)^\}", text, re.M | re.S):
        blocks, cur = {}, "entry"
        blocks[cur] = []
        for line in m.group(2).splitlines():
            label = re.match(r"([\w.$-]+):", line)
            if label:
                cur = label.group(1)
                blocks[cur] = []
            elif line.strip():
                blocks[cur].append(line.strip())
        yield m.group(1), blocks


def _arrays(blocks):
    """LDS arrays that each value may point into."""
    of, lines = {}, [l for b in blocks.values() for l in b]
    changed = True
    while changed:
        changed = False
        for l in lines:
            m = re.match(r"(%[\w.]+) = (?:getelementptr|phi|select|addrspacecast|bitcast|freeze)\b(.*)", l)
            if m:
                new = set(re.findall(r"@([\w.$]+)", m.group(2)))
                for v in re.findall(r"%[\w.]+", m.group(2)):
                    new |= of.get(v, set())
                if new - of.get(m.group(1), set()):
                    of[m.group(1)] = of.get(m.group(1), set()) | new
                    changed = True
    return of


def _access(line, of):
    """("store" | "load", arrays) of an LDS access, or None."""
    if re.search(r"\batomicrmw\b", line):
        return None                                  # (orders itself with the other lanes')
    m = re.search(r"\bstore (?:volatile )?.*?, ptr addrspace\(3\) (.*)", line) or \
        re.search(r"= load (?:volatile )?.*?, ptr addrspace\(3\) (.*)", line)
    if not m:
        return None
    arrays = set(re.findall(r"@([\w.$]+)", m.group(1)))
    first = re.match(r"%[\w.]+", m.group(1))
    arrays |= of.get(first.group(0), set()) if first else set()
    return ("load" if "= load" in line else "store"), arrays


def _unordered(blocks):
    of = _arrays(blocks)
    entry = {name: set() for name in blocks}         # accesses since the last fence: (kind, array)
    todo, seen, found, accesses = ["entry"], set(), set(), 0
    while todo:
        name = todo.pop()
        seen.add(name)
        since = set(entry[name])
        for line in blocks[name]:
            if line.startswith("fence ") or re.search(r"call void @llvm\.amdgcn\.s\.barrier\(", line):
                since = set()
            a = _access(line, of)
            if a:
                kind, arrays = a
                accesses += 1
                assert arrays, "an LDS access of no known array: " + line
                other = "load" if kind == "store" else "store"
                found |= {(x, other, kind) for x in arrays if (other, x) in since}
                since |= {(kind, x) for x in arrays}
        for target in re.findall(r"label %([\w.$-]+)", "\n".join(blocks[name])):
            if target not in seen or not since <= entry[target]:
                entry[target] |= since
                todo.append(target)
    return found, accesses


@pytest.mark.skipif(_hipcc() is None, reason="hipcc not available")
@pytest.mark.parametrize("source,kernels", [("hifa4_paged_decode.hip", ("k_runs_hif4",)),
                                            ("hifa4_paged.hip", ("k_paged_append",))])
def test_lanes_exchange_through_lds_in_order(source, kernels, tmp_path):
    seen = 0
    for name, blocks in _functions(_ir(source, tmp_path)):
        if any(k in name for k in kernels):
            found, accesses = _unordered(blocks)
            seen += accesses
            assert not found, f"{name}: {sorted(found)[:4]}"
    assert seen > 100, "nothing to check: the IR was not understood"


@pytest.mark.parametrize("lines,bad", [
    (["store i32 1, ptr addrspace(3) @a, align 4", "%1 = load i32, ptr addrspace(3) @a, align 4", "ret void"], True),
    (["store i32 1, ptr addrspace(3) @a, align 4", 'fence syncscope("wavefront") acq_rel', "%1 = load i32, ptr addrspace(3) @a, align 4",
      "ret void"], False),
    (["%1 = load i32, ptr addrspace(3) @a, align 4", "store i32 1, ptr addrspace(3) @a, align 4", "ret void"], True),
    (["%2 = getelementptr i32, ptr addrspace(3) @a, i32 %0", "store i32 1, ptr addrspace(3) %2, align 4",
      "%1 = load i32, ptr addrspace(3) @b, align 4", "ret void"], False),
])
def test_the_walk_finds_what_is_unordered(lines, bad):
    assert bool(_unordered({"entry": lines})[0]) == bad


def test_the_walk_follows_loops():
    loop = {"entry": ["br label %l"], "l": ["%1 = load i32, ptr addrspace(3) @a, align 4", "br i1 %c, label %m, label %e"],
            "m": ["store i32 1, ptr addrspace(3) @b, align 4", "br label %l"], "e": ["ret void"]}
    assert not _unordered(loop)[0]
    loop["m"][0] = loop["m"][0].replace("@b", "@a")
    assert _unordered(loop)[0] == {("a", "load", "store"), ("a", "store", "load")}
