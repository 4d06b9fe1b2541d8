"""CPU-only check of the numbers of mask words that the plan of a tree takes, with and without the request for every row."""
import ctypes as C
import os
import re

import pytest

from tests.test_paged_cpu import A, _cache, _refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


def test_words(mp):
    with open(os.path.join(ROOT, "include", "mp.h")) as f:
        assert int(re.search(r"#define MP_TREE_EVERY_ROW (\d+)", f.read()).group(1)) == mp.MP_TREE_EVERY_ROW
    c = _cache(mp)
    plan = lambda words, T=4: mp.lib().mp_paged_tree_plan(C.addressof(c), A, T, words, A + 4096, A + 512, None)      # noqa: E731
    for words in (0, 17, 255, -1, -256, -2 ** 31):
        _refused(mp, plan(words), "mask_words")
        _refused(mp, plan(words | mp.MP_TREE_EVERY_ROW), "mask_words")
    for words in (1, 16, 1 | mp.MP_TREE_EVERY_ROW, 16 | mp.MP_TREE_EVERY_ROW):
        assert plan(words, T=0) == mp.MP_OK
    # (other calls know no such request)
    _refused(mp, mp.lib().mp_paged_tree_keep(C.addressof(c), A, 1 | mp.MP_TREE_EVERY_ROW, 4, A + 512, A + 1024, None), "mask_words")
