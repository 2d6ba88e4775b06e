"""Properties of the built kernels that their sources are written for and a compiler may take away, read from the listing of the library's own
code.

Where registers are short, the compiler once stored some to the stack at the end of a branch that only some lanes take, while the others were
still switched off, and those got stale values back.  The walk of linear attention is short of registers, so nothing in it may switch lanes off.
"""
import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_10771_amd", "librslx.so")
OBJDUMP = os.environ.get("LLVM_OBJDUMP", "/opt/rocm/llvm/bin/llvm-objdump")
BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not installed")


def _code_objects(path):
    """The gfx950 code objects that the library carries, one for each source file."""
    data = open(path, "rb").read()
    at = data.find(BUNDLE)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(BUNDLE))
        p = at + len(BUNDLE) + 8
        for _ in range(count):
            offset, size, name = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + name].decode()
            p += 24 + name
            if "gfx950" in target and size:
                yield data[at + offset:at + offset + size]
        at = data.find(BUNDLE, at + 1)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Instructions of the sequence operators' kernels by mangled name."""
    out, where = {}, tmp_path_factory.mktemp("listing")
    for i, code in enumerate(_code_objects(LIB)):
        if b"walk_kernel" not in code and b"layer_norm_kernel" not in code:
            continue
        path = str(where / ("%d.co" % i))
        open(path, "wb").write(code)
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
        for line in text.split("\n"):
            head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if head:
                now = out[head.group(1)] = []
            elif line.startswith("\t"):
                now.append(line.split("//")[0].strip())
    return out


def test_the_walk_switches_no_lane_off(kernels):
    walks = {n: k for n, k in kernels.items() if "walk_kernel" in n}
    assert len(walks) > 100
    # what writes the mask: as an operation's destination, by saving and replacing it, or as a compare's result
    writes = re.compile(r"s_\w+ exec\b|s_\w+_saveexec|s_\w+_wrexec|v_cmpx")
    for name, code in walks.items():
        assert len(code) > 200
        found = [x for x in code if writes.match(x)]
        assert not found, (name, found[:3])


def test_the_other_kernels_keep_nothing_on_the_stack(kernels):
    others = {n: k for n, k in kernels.items() if "walk_kernel" not in n and ("norm" in n or "attention_step" in n or "walk_join" in n)}
    assert len(others) > 90
    for name, code in others.items():
        found = [x for x in code if x.startswith("scratch_") or "v_accvgpr" in x]
        assert not found, (name, len(found), found[0])
