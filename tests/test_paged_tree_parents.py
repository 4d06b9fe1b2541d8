"""CPU-only check of whom a token of a tree follows: a kernel keeps its parents in 16 bits, so whatever a caller passes has to come down to a token before it, or to -1."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_13059_amd", "csrc")


@pytest.fixture(scope="module")
def parent(tmp_path_factory):
    d = tmp_path_factory.mktemp("parent")
    src, so = d / "p.cpp", d / "p.so"
    src.write_text(f'''#include "{CSRC}/mp_page.h"
extern "C" int parent(int given, int token) {{ return (int16_t)mp::parent_of(given, token); }}
''')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(so), str(src)])
    return C.CDLL(str(so)).parent


@pytest.mark.parametrize("token", [0, 1, 6, 63, 64, 500, 1023])
def test_what_is_no_token_before_it_is_none(parent, token):
    given = list(range(-70, 1100)) + [s * (1 << 31) // 2 ** k + d for k in range(31) for s in (-1, 1) for d in (-1, 0, 1, 5, 1000)]
    for g in given:
        if -2 ** 31 <= g < 2 ** 31:
            assert parent(g, token) == (g if 0 <= g < token else -1), (g, token)


def test_the_kernel_asks_for_it():
    with open(os.path.join(CSRC, "mp_paged_tree.hip")) as f:
        kernel = f.read().split("void paged_tree_plan_kernel", 1)[1].split("\n}\n", 1)[0]
    assert kernel.count("parents[") == 1 and "parent_of(parents[" in kernel
