"""CPU-only check that results of trees and page tables that lie on what other workgroups of the same call still read, wholly or in part, are refused before the GPU is touched."""
import ctypes as C
import os

import pytest
import torch

from tests.test_paged_cpu import _refused

K, V, TABLE, LEN, START, IN, MASK, OUT = (1 << 20) * 1, (1 << 20) * 2, (1 << 20) * 3, (1 << 20) * 4, (1 << 20) * 5, (1 << 20) * 6, (1 << 20) * 7, (1 << 20) * 8
SEQS, TOKENS, WORDS, COLUMNS = 5, 40, 2, 9


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


def _cache(mp):
    return mp.MpPagedKvArgs(K, V, TABLE, LEN, START, 9, 16, 2, 128, SEQS, COLUMNS)


# (first byte, bytes) of what is read
READ = dict(kv_len=(LEN, 4 * SEQS), q_start=(START, 4 * SEQS + 4), parents=(IN, 4 * TOKENS), leaf=(IN, 4 * SEQS), mask=(MASK, 8 * TOKENS * WORDS), table=(TABLE, 4 * SEQS * COLUMNS))


def _on(what, size, step):
    """Addresses at which `size` bytes overlap it: its first and last elements' and, from before it, the last that reach into it."""
    at, n = READ[what]
    return [at, at + n - step, at - size + step]


@pytest.mark.parametrize("what", ["parents", "kv_len", "q_start"])
def test_plan(mp, what):
    c = _cache(mp)
    call = lambda mask, positions: mp.lib().mp_paged_tree_plan(C.addressof(c), IN, TOKENS, WORDS, mask, positions, None)      # noqa: E731
    for at in _on(what, 4 * TOKENS, 4):
        _refused(mp, call(MASK, at), "overlap")
    for at in _on(what, 8 * TOKENS * WORDS, 8):
        _refused(mp, call(at & ~7, OUT), "overlap")
    for at in _on("mask", 4 * TOKENS, 4):
        _refused(mp, call(MASK, at), "overlap")


@pytest.mark.parametrize("what", ["leaf", "mask", "kv_len", "q_start", "table"])
def test_keep(mp, what):
    c = _cache(mp)
    for at in _on(what, 4 * SEQS, 4):
        _refused(mp, mp.lib().mp_paged_tree_keep(C.addressof(c), MASK, WORDS, TOKENS, IN, at, None), "overlap")


def test_attention(mp):
    c = _cache(mp)
    call = lambda out, lse: mp.lib().mp_paged_tree_attention(C.addressof(c), IN, 0, MASK, WORDS, TOKENS, 4, 0, 0, 0.0, out, lse, K, 1 << 40, None)      # noqa: E731
    for at in _on("mask", 4 * TOKENS * 256, 16):
        _refused(mp, call(at, None), "overlaps the mask")
    for at in _on("mask", 4 * TOKENS * 4, 4):
        _refused(mp, call(OUT, at), "overlaps the mask")


@pytest.mark.parametrize("name", ["granted", "sequence", "positions", "slots"])
def test_reserve(mp, name):
    pool = mp.MpPagePoolArgs(TABLE, LEN, START, K, V, 9, 16, SEQS, COLUMNS)
    rows, keep = 11, OUT
    size, step = dict(granted=(4 * SEQS, 4), sequence=(4 * rows, 4), positions=(4 * rows, 4), slots=(8 * rows, 8))[name]
    others = [(LEN, 4 * SEQS), (START, 4 * SEQS + 4), (TABLE, 4 * SEQS * COLUMNS), (K, 36), (V, 4), (IN, 4 * SEQS), (keep, 4 * SEQS)]
    for at, n in others:
        for to in (at, at + n - 4, at - size + step):
            args = dict.fromkeys(("granted", "sequence", "positions", "slots"))
            args[name] = to & ~(step - 1)
            _refused(mp, mp.lib().mp_paged_reserve(C.addressof(pool), IN, keep, *args.values(), rows, None), "overlap")


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a GPU the launch itself fails")
def test_arrays_that_meet_do_not_overlap(mp):
    """Keys that stay right behind the lengths, and right before the starts."""
    c = _cache(mp)
    for keep in (LEN + 4 * SEQS, START - 4 * SEQS):
        assert mp.lib().mp_paged_tree_keep(C.addressof(c), MASK, WORDS, TOKENS, IN, keep, None) == mp.MP_EHIP


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a GPU the launch itself fails")
def test_no_rows_overlap_nothing(mp):
    pool = mp.MpPagePoolArgs(TABLE, LEN, START, K, V, 9, 16, SEQS, COLUMNS)
    for at in (START + 8, LEN, IN):
        assert mp.lib().mp_paged_reserve(C.addressof(pool), IN, None, None, at, None, None, 0, None) == mp.MP_EHIP
