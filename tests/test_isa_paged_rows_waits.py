"""CPU-only check that attention of trees with 33 to 128 query rows waits, while blocks go by, for nothing but its counted blocks: a wait of the compiler's own for a load to a register is one for
all loads to LDS before it.  (The counted waits themselves: test_isa_paged_rows.py.)"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_13059_amd import build
from tests.test_isa_paged_rows import SRC, _kernels


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_no_wait_but_those_for_blocks(tmp_path):
    asm = tmp_path / "rows.s"
    subprocess.check_call(["hipcc", *build.FLAGS, *build.EXTRA_FLAGS[os.path.basename(SRC)], "-S", "--cuda-device-only", "-o", str(asm), SRC], stderr=subprocess.DEVNULL)
    kernels = _kernels(asm.read_text().splitlines())
    assert set(kernels) == {(4, 0), (4, 1), (8, 0), (8, 1)}
    for (waves, one_page), lines in kernels.items():
        toks, in_asm = "", False
        for ln in lines:
            in_asm = ln.startswith(";;#ASMSTART") or (in_asm and not ln.startswith(";;#ASMEND"))
            if ln.startswith("global_load_lds_dwordx4"):
                toks += "L"                           # rows
            elif ln.startswith("global_load_lds_dword "):
                toks += "E"                           # entries of small pages
            elif re.match(r"(global|flat|buffer|scratch)_load", ln):
                toks += "g"                           # a load to registers
            elif ln.startswith("s_barrier"):
                toks += "B"
            elif "vmcnt(" in ln:
                toks += "W" if in_asm else "C"        # counted; the compiler's own
            elif ln.startswith("v_mfma"):
                toks += "M"
        assert toks.count("B") == 3, (waves, one_page)
        loads, loop = 64 // waves // 4 * 2, toks.split("B")[2]
        # a block's loads (small pages: entries before them), products, the loads of values that are not finite with their waits, the wait for the next block
        assert re.fullmatch(f"{'' if one_page else 'E'}L{{{loads}}}M+(g+C+)*W{{3}}", loop), (waves, one_page, re.sub(r"(.)\1+", r"\1+", loop))
