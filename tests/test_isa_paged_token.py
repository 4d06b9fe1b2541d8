"""CPU-only check of the load pipeline of attention over a paged cache for single tokens: its waves load straight to LDS and wait by count, so the
loads of a tile, compiled as they ship, have to stand in the order that the counts mean."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_13059_amd import build
from tests import test_isa_stream as ref

SRC = os.path.join(os.path.dirname(ref.SRC), "mp_paged_token.hip")


def _ends(blocks, label, at, stop):
    """{(keys read, loads to LDS, other accesses, the token stopped at)} of the ways on from a place; more than 40 of a kind are 40."""
    out, todo, visited = set(), [(label, at, 0, 0, 0)], set()
    while todo:
        state = todo.pop()
        if state in visited:
            continue
        visited.add(state)
        label, at, k, l, g = state
        toks, succ = blocks[label]
        for i in range(at, len(toks)):
            t = toks[i]
            if stop(t):
                out.add((k, l, g, t))
                break
            k, l, g = min(k + (t == "K"), 40), min(l + (t == "L16"), 40), min(g + (t == "G"), 40)
        else:
            todo += [(s, 0, k, l, g) for s in succ]
    return out


def _steps(blocks):
    """{(wait before the keys, loads to LDS and others up to the wait before the values, that wait)}, and the loads to LDS behind the values."""
    found, behind = set(), set()
    for label, (toks, _) in blocks.items():
        for i, t in enumerate(toks):
            if t.startswith("W"):
                for k, l, g, end in _ends(blocks, label, i + 1, lambda x: x.startswith("W") or x == "T"):
                    if k and end.startswith("W"):
                        assert k == 8, (k, l, g, end)
                        found.add((int(t[1:]), l, g, int(end[1:])))
            if t == "T" and toks[i:i + 8] == ["T"] * 8 and (i == 0 or toks[i - 1] != "T"):
                behind |= {l for _, l, _, _ in _ends(blocks, label, i, lambda x: x.startswith("W") or x == "G")}
    return found, behind


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_every_piece_has_arrived_before_its_use(tmp_path):
    asm = tmp_path / "token.s"
    subprocess.check_call(["hipcc", *build.FLAGS, *build.EXTRA_FLAGS.get(os.path.basename(SRC), []), "-S", "--cuda-device-only",
                           "-o", str(asm), SRC], stderr=subprocess.DEVNULL)
    text = re.sub(r"paged_token_kernelILi(\d)ELb(\d)E", r"value_stream_kernelILi\1ELi\2E", asm.read_text())
    checked = 0
    for groups, one_page, blocks in ref._kernels(text.splitlines()):
        found, behind = _steps(blocks)
        # two tiles or more follow: the keys of the one after next are asked for between the waits, and its pages' entries; one follows; none does
        main = [f for f in found if f[1]]
        rest = sorted((f for f in found if not f[1]), reverse=True)
        assert len(main) == 1 and main[0][1] == 8 and main[0][2] == 1, (groups, one_page, found)
        assert len(rest) == 2 and not any(f[2] for f in rest), (groups, one_page, found)
        assert behind <= {0, 8} and 8 in behind, (groups, one_page, behind)
        waits = {2: (main[0][0], main[0][3]), 1: (rest[0][0], rest[0][3]), 0: (rest[1][0], rest[1][3])}
        for n in range(1, 21):
            pending = [("entry", i) for i in range(4)] + [x for t in range(min(2, n)) for x in [("K", t)] * 8 + [("V", t)] * 8]

            def wait(most):
                del pending[:max(0, len(pending) - most)]
            for t in range(n):
                ahead = min(2, n - 1 - t)
                wait(waits[ahead][0])
                assert ("K", t) not in pending, (groups, one_page, n, t)
                if ahead == 2:
                    pending += [("K", t + 2)] * 8 + [("entry", t + 4)]
                wait(waits[ahead][1])
                assert ("V", t) not in pending, (groups, one_page, n, t)
                if ahead == 2:
                    pending += [("V", t + 2)] * 8
            assert not pending, (groups, one_page, n)
        checked += 1
    assert checked == 6
