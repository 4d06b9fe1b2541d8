"""CPU-only check that a batch of so many sequences that 32-bit counters would run past their end is refused by every call over a paged cache."""
import ctypes as C
import os

import pytest

from tests.test_paged_cpu import A, _cache, _refused


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("n_seqs", [2 ** 31 - 1024, 2 ** 31 - 64, 2 ** 31 - 1])
def test_too_many_sequences(mp, n_seqs):
    L, far = mp.lib(), A + (1 << 16)
    c = _cache(mp, n_seqs=n_seqs, table_stride=1)
    at = C.addressof(c)
    _refused(mp, L.mp_paged_append(at, None, None, 0, 0, None, A, 0, A, 0, 2, None), "too many sequences")
    _refused(mp, L.mp_paged_append_norm(at, None, None, None, A, None, 0, 0, None, A, 0, A, 0, 2, None), "too many sequences")
    _refused(mp, L.mp_paged_attention(at, A, 0, 2, 4, 0, 0, 0.0, far, None, A, 1 << 40, None), "too many sequences")
    _refused(mp, L.mp_paged_tree_attention(at, A, 0, A, 1, 2, 4, 0, 0, 0.0, far, None, A, 1 << 40, None), "too many sequences")
    _refused(mp, L.mp_paged_tree_plan(at, A, 2, 1, far, far + 4096, None), "sequences")
    _refused(mp, L.mp_paged_tree_keep(at, A, 1, 2, far, far + 4096, None), "too many")
    _refused(mp, L.mp_paged_gather(at, None, 0, 1, 0, A, None, None, None), "too many")
