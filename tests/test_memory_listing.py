"""Properties of the built kernels of the operators around a gated memory, read from the listing of the library's own code: nothing lies on the stack, where the
compiler has stored registers inside branches that only some lanes take."""
import os
import re
import subprocess

import pytest

from test_kernel_listing import LIB, OBJDUMP, _code_objects

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not installed")


def test_nothing_on_the_stack(tmp_path):
    seen = {}
    for i, code in enumerate(_code_objects(LIB)):
        if not any(n in code for n in (b"recurrence_kernel", b"rms_norm_kernel", b"muon_product_kernel")):
            continue
        path = str(tmp_path / ("%d.co" % i))
        open(path, "wb").write(code)
        name = None
        for line in subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout.split("\n"):
            head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if head:
                name = head.group(1)
            elif line.startswith("\t") and name:
                seen.setdefault(name, []).append(line.split("//")[0].strip())
    kernels = {n: k for n, k in seen.items() if "recurrence" in n or "rms_norm" in n or "muon" in n}
    for kind, least in (("recurrence_kernel", 20), ("recurrence_backward", 20), ("rms_norm_kernel", 90), ("rms_norm_backward", 45), ("muon_product", 8)):
        assert sum(kind in n for n in kernels) >= least, kind
    for name, code in kernels.items():
        found = [x for x in code if x.startswith("scratch_")]
        assert not found, (name, len(found), found[0])
