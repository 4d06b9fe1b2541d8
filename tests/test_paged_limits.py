"""CPU-only check of the table entries that attention over a paged cache asks for ahead, up to the longest sequence that a page table may have room for."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_13059_amd", "csrc")


@pytest.fixture(scope="module")
def entry(tmp_path_factory):
    d = tmp_path_factory.mktemp("entry")
    src, so = d / "e.cpp", d / "e.so"
    src.write_text(f'''#include "{CSRC}/mp_page.h"
extern "C" int entry(int block, int unit, int offset, int end, int shift) {{ return mp::entry_of(block, unit, offset, end, shift); }}
''')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(so), str(src)])
    return C.CDLL(str(so)).entry


@pytest.mark.parametrize("shift", [0, 1, 3, 4, 6, 7, 10])
def test_entries_asked_for_ahead_lie_in_the_sequence(entry, shift):
    """Tiles of 32 keys, up to four behind the last one (the token kernel's way of asking), of sequences of any length."""
    for end in (1, 2, 31, 32, 33, 1000, 2 ** 30 + 5, 2 ** 31 - 161, 2 ** 31 - 129, 2 ** 31 - 128, 2 ** 31 - 64, 2 ** 31 - 2, 2 ** 31 - 1):
        last = (end - 1) // 32
        for tile in range(max(0, last - 2), last + 5):
            for offset in (0, 16, 31):
                assert entry(tile, 32, offset, end, shift) == min(tile * 32 + offset, end - 1) >> shift, (end, tile, offset)


def test_the_token_kernel_asks_in_this_way():
    with open(os.path.join(CSRC, "mp_paged_token.hip")) as f:
        line = next(x for x in f if "auto entry_at" in x)
    assert "entry_of(t, kTile," in line
