"""CPU-only check of the load pipeline of attention of trees with 33 to 128 query rows: its waves load straight to LDS and wait by count, so the loads of a block, compiled as they
ship, have to be as many as the counts mean, and waits have to be those of blocks that are still on their way."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_13059_amd import build

SRC = os.path.join(build.CSRC, "mp_paged_rows.hip")


def _kernels(asm):
    """{(waves, one page): lines} of every kernel."""
    out, cur = {}, None
    for ln in asm:
        m = re.match(r"^_ZN2mp\S*paged_tree_rows_kernelILi(\d+)ELb(\d)E\S*:", ln)
        if m:
            cur = out.setdefault((int(m.group(1)), int(m.group(2))), [])
        elif ln.startswith(".Lfunc_end"):
            cur = None
        elif cur is not None:
            cur.append(ln.strip())
    return out


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_blocks_are_waited_for_by_their_loads(tmp_path):
    asm = tmp_path / "rows.s"
    subprocess.check_call(["hipcc", *build.FLAGS, *build.EXTRA_FLAGS[os.path.basename(SRC)], "-S", "--cuda-device-only", "-o", str(asm), SRC], stderr=subprocess.DEVNULL)
    kernels = _kernels(asm.read_text().splitlines())
    assert set(kernels) == {(4, 0), (4, 1), (8, 0), (8, 1)}
    for (waves, one_page), lines in kernels.items():
        loads = 64 // waves // 4 * 2                  # of a block, a wave: four rows an instruction, keys and values
        toks, in_asm = [], False
        for ln in lines:
            in_asm = ln.startswith(";;#ASMSTART") or (in_asm and not ln.startswith(";;#ASMEND"))
            if ln.startswith("global_load_lds_dwordx4"):
                toks.append("L")
            elif ln.startswith("s_barrier"):
                toks.append("B")
            elif in_asm and re.match(r"s_waitcnt vmcnt\(\d+\)", ln):
                toks.append(int(re.search(r"vmcnt\((\d+)\)", ln).group(1)))
            elif ln.startswith("scratch_"):
                toks.append("S")
            elif ln.startswith("v_mfma"):
                toks.append("M")
        assert "S" not in toks, (waves, one_page)
        # loads stand in runs of whole blocks: three in front of the loop and one in it
        assert toks.count("L") == 4 * loads, (waves, one_page)
        # a block's wait leaves two blocks on their way, one, or none; in front of the loop and at its end
        waits = [t for t in toks if isinstance(t, int)]
        assert sorted(waits) == sorted(2 * [0, loads, 2 * loads]), (waves, one_page, waits)
        # in order: an item begins where all have met, three blocks, the first one's wait, all meet, one block more, products, the next one's wait, all meet
        order = "".join("W" if isinstance(t, int) else t for t in toks)
        assert re.fullmatch(f"BL{{{3 * loads}}}W{{3}}BL{{{loads}}}M+W{{3}}B", order), (waves, one_page, re.sub(r"(.)\1+", r"\1+", order))
