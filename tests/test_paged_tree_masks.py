"""CPU-only check of which keys a token of a tree attends, against sets of numbers, up to the longest sequence that a page table may have room for."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_13059_amd", "csrc")


@pytest.fixture(scope="module")
def tree(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree")
    src, so = d / "t.cpp", d / "t.so"
    src.write_text(f'''#include "{CSRC}/mp_page.h"
extern "C" int low(const unsigned long long* mask, int words, int base, int n, int window) {{ return mp::tree_low(mask, words, base, n, window); }}
extern "C" unsigned long long keys(const unsigned long long* mask, int words, int low, int base, int first) {{ return mp::tree_keys(mask, words, low, base, first); }}
''')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(so), str(src)])
    h = C.CDLL(str(so))
    h.keys.restype = C.c_ulonglong
    return h


@pytest.mark.parametrize("far", [0, 2 ** 31 - 1 - 64 * 40])
def test_keys_of_a_row(tree, far):
    rng = np.random.default_rng(7)
    for _ in range(4000):
        n, words = int(rng.integers(1, 200)), int(rng.integers(1, 5))
        base = far + int(rng.integers(-n, 900))
        window = int(rng.choice([0, 1, 2, 5, 40, 64, 65, 130, 700, 2 ** 31 - 1]))
        marks = [i for i in range(64 * words) if rng.random() < rng.choice([0.0, 0.1, 0.6, 1.0])]
        mask = (C.c_ulonglong * words)(*[sum(1 << (i % 64) for i in marks if i // 64 == w) for w in range(words)])
        end = base + n                                              # what lies behind is no key
        older_from = max(0, base - 800) if far else 0
        attended = list(range(older_from, max(base, 0))) + [base + i for i in marks if i < n]
        if window:
            attended = attended[-window:]
        attended = set(attended)
        low = tree.low(mask, words, base, n, window)
        if window == 0:
            assert low == 0
        for block in range(max(0, base - 200) // 64, (end + 63) // 64):
            got = tree.keys(mask, min(words, (n + 63) // 64), low, base, block * 64)
            for k in range(64):
                key = block * 64 + k
                if key < end and (window < 600 or not far):
                    assert (got >> k & 1) == (key in attended), (base, n, words, window, key)


def test_a_window_larger_than_all_keys_leaves_all(tree):
    mask = (C.c_ulonglong * 1)(5)
    assert tree.low(mask, 1, 100, 3, 2 ** 31 - 1) == 0 and tree.low(mask, 1, -2, 3, 7) == 0 and tree.low(mask, 1, 2 ** 31 - 70, 3, 4) == 2 ** 31 - 72
