"""CPU-only checks of rotary positions and the paged cache: frequencies, where a key lies, and what is refused before the GPU is touched."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_13059_amd", "csrc")


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("rot,base", [(128, 1e4), (64, 5e5), (2, 1e4), (20, 1e6)])
def test_frequencies(mp, rot, base):
    i = np.arange(rot // 2)
    plain = base ** (-2.0 * i / rot)
    np.testing.assert_allclose(mp.mp_rotary_frequencies(rot, base).numpy(), plain, rtol=1e-14)
    np.testing.assert_allclose(mp.mp_rotary_frequencies(rot, base, mp.MP_ROTARY_LINEAR, 4.0).numpy(), plain / 4, rtol=1e-14)
    if rot > 2:
        # the slowest pair of the scaled base is the plain one slowed down by the factor, the fastest stays
        f = mp.mp_rotary_frequencies(rot, base, mp.MP_ROTARY_BASE, 8.0).numpy()
        np.testing.assert_allclose([f[0], f[-1]], [1.0, plain[-1] / 8], rtol=1e-13)
    f = mp.mp_rotary_frequencies(rot, base, mp.MP_ROTARY_BY_PARTS, 4.0, 8192, 1.0, 32.0).numpy()
    turns = 8192 * plain / (2 * math.pi)
    for k in range(rot // 2):
        if turns[k] >= 32:
            assert abs(f[k] / plain[k] - 1) < 1e-14
        elif turns[k] <= 1:
            assert abs(f[k] / plain[k] - 0.25) < 1e-14
        else:
            g = (turns[k] - 1) / 31
            assert abs(f[k] - (g * plain[k] + (1 - g) * plain[k] / 4)) < 1e-14


@pytest.mark.parametrize("args", [(0,), (3,), (130,), (64, 0.0), (64, math.nan), (64, 1e4, 4), (64, 1e4, -1), (64, 1e4, 1, 0.0), (2, 1e4, 2, 2.0),
                                  (64, 1e4, 3, 4.0, 0.0), (64, 1e4, 3, 4.0, 8192.0, 32.0, 1.0), (64, 1e4, 1, math.inf)])
def test_frequencies_refuse(mp, args):
    with pytest.raises(mp.MpError) as e:
        mp.mp_rotary_frequencies(*args)
    assert e.value.status == mp.MP_EINVAL
    assert mp.lib().mp_rotary_frequencies(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == mp.MP_EINVAL


@pytest.fixture(scope="module")
def where(tmp_path_factory):
    d = tmp_path_factory.mktemp("page")
    src, so = d / "p.cpp", d / "p.so"
    src.write_text(f'''#include "{CSRC}/mp_page.h"
extern "C" int page(const int* row, int stride, int n_pages, int shift, int position) {{ return mp::page_of(row, stride, n_pages, shift, position); }}
extern "C" long long row(int page, int head, int n_kv, int shift, int position) {{ return mp::row_of(page, head, n_kv, shift, position); }}
''')
    src.write_text(src.read_text() + '''
extern "C" void blocks(int base, int i0, int i1, int window, int room, int unit, int* out) { mp::blocks_of(base, i0, i1, window, room, unit, out, out + 1); }
extern "C" void parts(long long x0, long long x1, long long share, long long* out)
{
    const mp::Parts p = mp::parts_of(x0, x1, share);
    out[0] = p.first;
    out[1] = p.last;
}
extern "C" int slot(long long x0, long long workgroup, long long share) { return mp::slot_of(x0, workgroup, share); }
''')
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-o", str(so), str(src)])
    h = C.CDLL(str(so))
    h.row.restype = C.c_longlong
    h.parts.argtypes = [C.c_longlong] * 3 + [C.POINTER(C.c_longlong)]
    h.slot.argtypes = [C.c_longlong] * 3
    return h


def test_pages_that_are_not_there(where):
    row = (C.c_int * 4)(5, -1, 7, 2)
    got = [where.page(row, 4, 7, 4, p) for p in (0, 15, 16, 31, 32, 48, 63, 64, 1 << 30, -1, -17, -(1 << 31))]
    assert got == [5, 5, -1, -1, -1, 2, 2, -1, -1, -1, -1, -1]      # (entry 7 of 7 pages: out of range)
    assert where.page(row, 4, 8, 4, 32) == 7 and where.page(row, 4, 7, 0, 3) == 2


def test_rows_pass_32_bits(where):
    assert where.row(3, 1, 2, 4, 37) == (3 * 2 + 1) * 16 + 5
    assert where.row(2 ** 31 - 1, 7, 8, 10, 2 ** 31 - 1) == (((2 ** 31 - 1) * 8 + 7) << 10) + 1023


def test_blocks_are_those_of_the_keys_that_are_attended(where):
    rng = np.random.default_rng(3)
    out = (C.c_int * 2)()
    for _ in range(3000):
        unit, n = int(rng.choice([64, 128])), int(rng.integers(1, 60))
        length, window = int(rng.integers(0, 900)), int(rng.choice([0, 0, 1, 37, 300]))
        base, room = length - n, int(rng.choice([1 << 20, 300, 64]))
        i0 = int(rng.integers(0, n))
        i1 = int(rng.integers(i0, n))
        keys = [j for i in (i0, i1) for j in range(max(0, base + i - window + 1) if window else 0, min(base + i + 1, room))]
        where.blocks(base, i0, i1, window, room, unit, out)
        assert out[1] > out[0] >= 0
        if keys:
            assert out[0] * unit <= min(keys) and max(keys) < out[1] * unit
            assert min(keys) < (out[0] + 1) * unit and max(keys) >= (out[1] - 1) * unit      # (and no more)
    where.blocks(2 ** 31 - 1 - 8, 0, 7, 0, 2 ** 31 - 1, 64, out)
    assert list(out) == [0, 2 ** 25]


def test_parts_of_items_have_places_of_their_own(where):
    # items one after another on a line that is cut into shares: every block of an item lies in one of its parts, and no two parts of different items share a slot
    rng = np.random.default_rng(4)
    out = (C.c_longlong * 2)()
    for _ in range(300):
        share, ahead, x, used = int(rng.integers(1, 40)), int(rng.integers(0, 4)), 0, {}
        for item in range(40):
            x0 = x + ahead
            x = x1 = x0 + int(rng.integers(1, 90))
            where.parts(x0, x1, share, out)
            first, last = out[0], out[1]
            assert first * share <= x0 < (first + 1) * share and last * share < x1 <= (last + 1) * share
            if first == last:
                continue
            for g in range(first, last + 1):
                at = g, where.slot(x0, g, share)
                assert at[1] == (0 if g > first else int(x0 > g * share)) and at not in used
                used[at] = item


# (addresses that no one reads: every call is refused before a launch)
A = 1 << 20


def _spec(mp, **kw):
    d = dict(freqs=A, rot_dim=128, layout=0, amplitude=1.0)
    d.update(kw)
    return mp.MpRotarySpec(*d.values())


def _cache(mp, **kw):
    d = dict(k_pages=A, v_pages=A, page_table=A, kv_len=A, q_start=A, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, n_seqs=1, table_stride=4)
    d.update(kw)
    return mp.MpPagedKvArgs(*d.values())


def _refused(mp, status, word=None):
    assert status == mp.MP_EINVAL
    if word:
        assert word.encode() in mp.lib().mp_last_error(None)


def test_rotary_refuses(mp):
    call = lambda spec, x=A, xs=0, pos=A, T=2, H=3, out=A + 4096, os_=0, look=None: mp.lib().mp_rotary(      # noqa: E731
        None if spec is None else C.addressof(spec), x, xs, pos, T, H, out, os_, look, 0, None)
    ok = _spec(mp)
    _refused(mp, call(None), "null rotary")
    for kw in (dict(freqs=None), dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=130), dict(layout=2), dict(amplitude=math.inf), dict(amplitude=math.nan)):
        _refused(mp, call(_spec(mp, **kw)), "mp_rotary")
    _refused(mp, call(ok, x=None), "null x")
    _refused(mp, call(ok, x=A + 8), "16 bytes")
    _refused(mp, call(ok, pos=None), "positions")
    _refused(mp, call(ok, out=None), "no output")
    _refused(mp, call(ok, out=A + 4098), "16 bytes")
    _refused(mp, call(ok, xs=3 * 128 - 8), "stride")
    _refused(mp, call(ok, xs=3 * 128 + 4), "stride")
    _refused(mp, call(ok, os_=100), "stride")
    _refused(mp, call(ok, T=-1), "sizes")
    _refused(mp, call(ok, H=0), "sizes")
    _refused(mp, call(ok, out=A, xs=512), "in place")
    _refused(mp, call(ok, look=A + 4096), "overlaps")
    _refused(mp, call(ok, out=None, xs=512, look=A), "overlaps")
    assert call(ok, T=0) == mp.MP_OK


BAD_CACHES = [dict(k_pages=None), dict(v_pages=A + 2), dict(page_table=None), dict(kv_len=None), dict(q_start=None), dict(n_pages=0), dict(page_size=0),
              dict(page_size=24), dict(page_size=2048), dict(n_kv_heads=0), dict(head_dim=64), dict(n_seqs=-1), dict(table_stride=0),
              dict(page_size=1024, table_stride=1 << 21)]


def test_append_refuses(mp):
    call = lambda c, spec=None, q=None, qs=0, hq=0, qo=None, k=A, ks=0, v=A, vs=0, T=2: mp.lib().mp_paged_append(      # noqa: E731
        None if c is None else C.addressof(c), None if spec is None else C.addressof(spec), q, qs, hq, qo, k, ks, v, vs, T, None)
    ok = _cache(mp)
    _refused(mp, call(None), "null cache")
    for kw in BAD_CACHES:
        _refused(mp, call(_cache(mp, **kw)), "mp_paged_append")
    _refused(mp, call(ok, spec=_spec(mp, rot_dim=5)), "rot_dim")
    _refused(mp, call(ok, q=A), "together")
    _refused(mp, call(ok, qo=A), "together")
    _refused(mp, call(ok, q=A, qo=A, hq=0), "n_q_heads")
    _refused(mp, call(ok, q=A, qo=A, hq=2, qs=512), "in place")
    _refused(mp, call(ok, q=A, qo=A + 2, hq=2), "16 bytes")
    _refused(mp, call(ok, k=None), "null k")
    _refused(mp, call(ok, vs=248), "stride")
    _refused(mp, call(ok, T=-1), "n_tokens")
    assert call(ok, T=0) == mp.MP_OK and call(_cache(mp, n_seqs=0)) == mp.MP_OK


def test_gather_refuses(mp):
    call = lambda c, spec=None, first=0, n=3, k=A, kl=None, v=A: mp.lib().mp_paged_gather(      # noqa: E731
        None if c is None else C.addressof(c), None if spec is None else C.addressof(spec), first, n, 0, k, kl, v, None)
    ok = _cache(mp)
    _refused(mp, call(None), "null cache")
    for kw in BAD_CACHES:
        _refused(mp, call(_cache(mp, **kw)), "mp_paged_gather")
    _refused(mp, call(ok, kl=A), "null rotary")
    _refused(mp, call(ok, first=-1), "range")
    _refused(mp, call(ok, n=-1), "range")
    _refused(mp, call(ok, first=2 ** 31 - 2, n=3), "range")
    _refused(mp, call(ok, k=None, v=None), "no output")
    _refused(mp, call(ok, v=A + 8), "16 bytes")
    assert call(ok, n=0) == mp.MP_OK


def test_attention_refuses(mp):
    def call(c, q=A, qs=0, T=2, hq=8, most=0, window=0, scale=0.0, out=A, lse=None, ws=A, bytes_=1 << 40):
        return mp.lib().mp_paged_attention(None if c is None else C.addressof(c), q, qs, T, hq, most, window, scale, out, lse, ws, bytes_, None)
    ok = _cache(mp)
    _refused(mp, call(None), "null cache")
    for kw in BAD_CACHES:
        _refused(mp, call(_cache(mp, **kw)), "mp_paged_attention")
    for kw in (dict(T=-1), dict(hq=0), dict(hq=7), dict(hq=18), dict(most=-1), dict(window=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
               dict(q=None), dict(q=A + 2), dict(qs=8), dict(out=None), dict(out=A + 4), dict(ws=A + 4)):
        _refused(mp, call(ok, **kw), "mp_paged_attention")
    need = mp.mp_paged_workspace_bytes(2, 8, 2, 1, 0)
    if need:
        _refused(mp, call(ok, bytes_=need - 1), "workspace")
        _refused(mp, call(ok, ws=None), "workspace")
    assert call(ok, T=0) == mp.MP_OK and call(_cache(mp, n_seqs=0)) == mp.MP_OK
    assert mp.mp_paged_workspace_bytes(2, 7, 2, 1, 1) == mp.mp_paged_workspace_bytes(-1, 8, 2, 1, 1) == mp.mp_paged_workspace_bytes(2, 18, 2, 1, 1) == 0


def test_rows_that_lie_over_one_another_are_refused(mp):
    """A broadcast token has no stride, which the library would take for densely packed rows: past the tensor's end."""
    import torch
    x = torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    for bad in (x.expand(4, 2, 128), torch.zeros(900, dtype=torch.bfloat16).as_strided((3, 2, 128), (128, 128, 1))):
        with pytest.raises(mp.MpError) as e:
            mp._token_rows(bad, "x", bad.get_device())
        assert e.value.status == mp.MP_EINVAL
    assert mp._token_rows(x, "x", x.get_device()) == (1, 2, 0)
    assert mp._token_rows(x.expand(4, 2, 128).contiguous(), "x", x.get_device()) == (4, 2, 256)
    assert mp._token_rows(torch.zeros(4, 5, 128, dtype=torch.bfloat16)[:, 1:3], "x", -1) == (4, 2, 640)


def test_attention_does_not_write_over_its_queries(mp):
    """Workgroups that share a tile of rows read its queries until the last of them is done."""
    cache = _cache(mp)

    def call(q, out, qs=0):
        return mp.lib().mp_paged_attention(C.addressof(cache), q, qs, 2, 8, 0, 0, 0.0, out, None, A, 1 << 40, None)
    rows = 8 * 128 * 2
    for q, out, qs in ((A, A, 0), (A, A + 2 * rows - 16, 0), (A + 2 * rows - 16, A, 0), (A, A + 3 * rows, 8 * 128 * 4), (A, A + rows, 8 * 128 * 4)):
        _refused(mp, call(q, out, qs), "overlaps")


def test_launches_and_lines_that_pass_their_counters_are_refused(mp):
    """A launch counts its lanes and a line of blocks its places in 32 bits."""
    spec, wide = _spec(mp), _cache(mp, page_size=1024, table_stride=(1 << 21) - 1)
    many = 1 << 27
    _refused(mp, mp.lib().mp_rotary(C.addressof(spec), A, 0, A, many, 1, A, 0, None, 0, None), "too many")
    cache = _cache(mp)
    _refused(mp, mp.lib().mp_paged_append(C.addressof(cache), None, None, 0, 0, None, A, 0, A, 0, many, None), "too many")
    lots = _cache(mp, n_seqs=1 << 20)
    _refused(mp, mp.lib().mp_paged_gather(C.addressof(lots), None, 0, 4096, 0, A, None, A, None), "too many")
    out = A + (1 << 50)
    attend = lambda c, T, hq, most=0, window=0: mp.lib().mp_paged_attention(C.addressof(c), A, 0, T, hq, most, window, 0.0, out, None, A, 1 << 40, None)      # noqa: E731
    _refused(mp, attend(wide, 1 << 20, 16), "too many")                                         # 2^31 keys under each of 2^15 tiles
    for kw in (dict(n_seqs=1 << 17), dict(n_seqs=1 << 20)):                                     # 2^31 keys of each of many sequences
        c = _cache(mp, page_size=1024, table_stride=(1 << 21) - 1, **kw)
        _refused(mp, attend(c, kw["n_seqs"], 2, 1), "too many")
    _refused(mp, attend(wide, 1 << 20, 16, window=1 << 30), "too many")
