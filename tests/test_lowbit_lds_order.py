"""Where lanes hand data to each other through LDS, the compiler has to be told: to it a lane's stores and its loads of other lanes'
data are unrelated.  Read off the intermediate code that the 4-bit linear kernels' source compiles to: on no path may a load from LDS
follow a store to it, or a store a load, without a fence between them (a barrier has one on both sides)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2405_05329_amd import build as kbuild

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


def functions(text):
    """{name: {label: ([instruction, ...], [successor, ...])}} of a module; the first block of a function is called "entry"."""
    out = {}
    for m in re.finditer(r"^define [^\n]*@([\w.$]+)\([^\n]*\{\n(.*?)^\}", text, re.M | re.S):
        blocks, label = {"entry": ([], [])}, "entry"
        for line in m[2].splitlines():
            head = re.match(r"^([\w.$]+):", line)
            if head:
                label = head[1]
                blocks[label] = ([], [])
            elif line.strip():
                blocks[label][0].append(line.strip())
                blocks[label][1].extend(re.findall(r"label %([\w.$]+)", line))
        out[m[1]] = blocks
    return out


def touches(line):
    """'load' or 'store' of LDS, 'fence', or None."""
    if re.match(r"(tail |musttail |notail )?fence\b", line) or ("asm sideeffect" in line and "~{memory}" in line):
        return "fence"
    if line.startswith("store ") and "ptr addrspace(3)" in line:
        return "store"
    if re.match(r"%[\w.]+ = load ", line) and "ptr addrspace(3)" in line:
        return "load"
    return None


def unordered(blocks):
    """Instructions that meet the other kind of LDS access on some path since the last fence."""
    arriving, found = {label: set() for label in blocks}, set()
    todo = ["entry"]
    seen = set()
    while todo:
        label = todo.pop()
        seen.add(label)
        since = set(arriving[label])
        for line in blocks[label][0]:
            kind = touches(line)
            if kind == "fence":
                since.clear()
            elif kind:
                if since - {kind}:
                    found.add(line)
                since.add(kind)
        for nxt in blocks[label][1]:
            if nxt not in seen or not since <= arriving[nxt]:
                arriving[nxt] |= since
                todo.append(nxt)
    return found


@pytest.fixture(scope="module")
def w4(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("ir") / "w4.ll")
    subprocess.run([HIPCC, "-O3", "-std=c++17", "-fPIC", "-I", os.path.join(kbuild.ROOT, "include"), "-I", kbuild.CSRC, *kbuild.DEVICE_FLAGS,
                    *kbuild.FILE_FLAGS.get("kvra_w4.hip", []), "-x", "hip", "--cuda-device-only", "-S", "-emit-llvm",
                    os.path.join(kbuild.CSRC, "kvra_w4.hip"), "-o", path], check=True, capture_output=True)
    with open(path) as f:
        return functions(f.read())


@pytest.mark.parametrize("kernel,count", [("linear_w4_rows_kernel", 8), ("linear_w4_tile_kernel", 4)])
def test_lds_is_handed_over_in_order(w4, kernel, count):
    mine = {name: blocks for name, blocks in w4.items() if kernel in name}
    assert len(mine) == count
    for name, blocks in mine.items():
        kinds = [touches(line) for lines, _ in blocks.values() for line in lines]
        assert kinds.count("load") >= 8 and kinds.count("fence") >= 2, name      # (nothing is there only if the text is not understood)
        found = unordered(blocks)
        assert not found, (name, len(found), sorted(found)[:2])


def test_the_check_sees_what_it_is_for():
    body = """define void @f(i1 %c) {{
  br label %loop

loop:                                             ; preds = %loop, %0
  {first}store <4 x i32> %a, ptr addrspace(3) %p, align 16
  {second}%x = load <4 x i32>, ptr addrspace(3) %q, align 16
  store i32 %y, ptr addrspace(1) %g, align 4
  br i1 %c, label %loop, label %done

done:
  ret void
}}
"""
    fence = 'fence syncscope("wavefront") release\n  '
    count = lambda first, second: len(unordered(functions(body.format(first=first, second=second))["f"]))
    assert [count("", ""), count(fence, ""), count("", fence), count(fence, fence)] == [2, 1, 1, 0]
