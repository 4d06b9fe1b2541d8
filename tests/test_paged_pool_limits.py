"""CPU-only check of the sizes that a step of page tables is refused for: its kernels count rows and sequences in 32 bits."""
import ctypes as C
import os

import pytest

from tests.test_paged_cpu import A, _refused


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("kw", [dict(rows=2 ** 31 - 1), dict(rows=2 ** 31 - 64), dict(n_seqs=2 ** 31 - 1, table_stride=1), dict(n_seqs=2 ** 31 - 1024, table_stride=1)])
def test_steps_past_32_bits_are_refused(mp, kw):
    d = dict(rows=5, n_seqs=2, table_stride=4) | kw
    pool = mp.MpPagePoolArgs(A, A + 1024, A + 2048, A + 4096, A + 8192, 9, 16, d["n_seqs"], d["table_stride"])
    _refused(mp, mp.lib().mp_paged_reserve(C.addressof(pool), A + 64, None, None, A + 512, None, None, d["rows"], None), "too many rows or sequences")
