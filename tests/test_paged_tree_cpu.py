"""CPU-only checks of what norms, page pools and trees refuse before the GPU is touched."""
import ctypes as C
import math
import os

import pytest

from tests.test_paged_cpu import A, BAD_CACHES, _cache, _refused, _spec


@pytest.fixture(scope="module")
def mp():
    from paper_2506_13059_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


def _norm(mp, **kw):
    d = dict(weight=A, n_heads=1, offset=0.0, eps=1e-6)
    d.update(kw)
    return mp.MpHeadNormSpec(*d.values())


def _at(x):
    return None if x is None else C.addressof(x)


BAD_NORMS = [dict(weight=None), dict(weight=A + 8), dict(n_heads=0), dict(n_heads=2), dict(n_heads=-1), dict(offset=math.nan), dict(eps=0.0), dict(eps=-1e-6), dict(eps=math.inf),
             dict(eps=math.nan)]


def test_norm_rotary_refuses(mp):
    def call(norm, spec=_spec(mp), x=A, xs=0, pos=A, T=2, H=3, out=A + 4096, os_=0, look=None):
        return mp.lib().mp_norm_rotary(_at(norm), _at(spec), x, xs, pos, T, H, out, os_, look, 0, None)
    ok = _norm(mp)
    _refused(mp, call(None), "null norm")
    for kw in BAD_NORMS:
        _refused(mp, call(_norm(mp, **kw)), "mp_norm_rotary")
        _refused(mp, call(_norm(mp, **kw), T=0), "mp_norm_rotary")
    _refused(mp, call(ok, spec=None), "mp_norm_rotary: null rotary")
    _refused(mp, call(ok, spec=_spec(mp, rot_dim=7)), "rot_dim")
    _refused(mp, call(ok, x=None), "null x")
    _refused(mp, call(ok, pos=None), "positions")
    _refused(mp, call(ok, out=None), "no output")
    _refused(mp, call(ok, xs=3 * 128 - 8), "stride")
    _refused(mp, call(ok, out=A, xs=512), "in place")
    _refused(mp, call(ok, look=A + 4096), "overlaps")
    _refused(mp, call(ok, T=1 << 30), "too many")
    assert call(ok, T=0) == mp.MP_OK and call(_norm(mp, n_heads=3), T=0) == mp.MP_OK


def test_append_norm_refuses(mp):
    def call(cache=_cache(mp), spec=_spec(mp), qn=None, kn=None, q=A, qs=0, Hq=4, qo=A, k=A, ks=0, v=A, vs=0, T=3):
        return mp.lib().mp_paged_append_norm(_at(cache), _at(spec), _at(qn), _at(kn), None, q, qs, Hq, qo, k, ks, v, vs, T, None)
    for kw in BAD_CACHES:
        _refused(mp, call(_cache(mp, **kw)), "mp_paged_append_norm")
    for kw in BAD_NORMS:
        _refused(mp, call(qn=_norm(mp, **kw)), "of q")
        assert call(qn=_norm(mp, **kw), q=None, qo=None, T=0) == mp.MP_OK          # (not looked at without q)
    for kw in BAD_NORMS[:3] + BAD_NORMS[4:]:
        _refused(mp, call(kn=_norm(mp, **kw)), "of k")
    _refused(mp, call(kn=_norm(mp, n_heads=3)), "of k")
    _refused(mp, call(qo=None), "together")
    _refused(mp, call(k=None), "null k")
    _refused(mp, call(vs=130), "stride")
    _refused(mp, call(q=A, qs=1024), "in place")
    assert call(qn=_norm(mp, n_heads=4), kn=_norm(mp, n_heads=2), T=0) == mp.MP_OK


def test_reserve_refuses(mp):
    def call(n_new=A + 64, keep=None, granted=None, sequence=None, positions=None, slots=None, rows=0, null=False, **kw):
        d = dict(page_table=A, kv_len=A + 1024, q_start=A + 2048, free_pages=A + 4096, n_free=A + 8192, n_pages=9, page_size=16, n_seqs=2, table_stride=4)
        d.update(kw)
        pool = mp.MpPagePoolArgs(*d.values())
        return mp.lib().mp_paged_reserve(None if null else C.addressof(pool), n_new, keep, granted, sequence, positions, slots, rows, None)
    _refused(mp, call(null=True), "null pool")
    for kw in (dict(n_pages=0), dict(n_seqs=-1), dict(table_stride=0), dict(page_size=0), dict(page_size=24), dict(page_size=2048), dict(page_size=1024, table_stride=1 << 21),
               dict(page_size=1024, n_pages=1 << 21), dict(n_seqs=1 << 20, table_stride=1 << 11), dict(page_table=None), dict(kv_len=None), dict(q_start=None),
               dict(free_pages=None), dict(n_free=None), dict(n_new=None), dict(rows=-1), dict(slots=A + 516)):
        _refused(mp, call(**kw), "mp_paged_reserve")
    for kw in (dict(n_new=A + 1024), dict(keep=A + 1024), dict(keep=A + 512, granted=A + 512), dict(granted=A + 64), dict(granted=A + 512, positions=A + 512),
               dict(sequence=A + 2048), dict(slots=A + 512, positions=A + 512)):
        _refused(mp, call(rows=5, **kw), "overlap")


def test_trees_refuse(mp):
    L = mp.lib()
    plan = lambda c=_cache(mp), p=A, T=4, W=1, m=A, pos=A + 512: L.mp_paged_tree_plan(C.addressof(c), p, T, W, m, pos, None)      # noqa: E731
    keep = lambda c=_cache(mp), m=A, W=1, T=4, leaf=A + 512, k=A + 1024: L.mp_paged_tree_keep(C.addressof(c), m, W, T, leaf, k, None)      # noqa: E731
    attend = lambda c=_cache(mp), q=A, qs=0, m=A, W=1, T=4, Hq=8, new=2, window=0, scale=0.0, out=A + (1 << 16), ws=A, size=1 << 40: L.mp_paged_tree_attention(      # noqa: E731
        C.addressof(c), q, qs, m, W, T, Hq, new, window, scale, out, None, ws, size, None)
    for name, call in (("plan", plan), ("keep", keep), ("attention", attend)):
        for kw in BAD_CACHES:
            _refused(mp, call(_cache(mp, **kw)), "mp_paged_tree_" + name)
        for kw in (dict(W=0), dict(W=17), dict(m=None), dict(m=A + 4), dict(T=-1)):
            _refused(mp, call(**kw), "mp_paged_tree_" + name)
    _refused(mp, plan(p=None), "null parents")
    _refused(mp, plan(pos=None), "null parents")
    _refused(mp, plan(p=A + 512), "overlap")
    _refused(mp, plan(_cache(mp, n_seqs=1 << 22)), "sequences")
    _refused(mp, keep(leaf=None), "null leaf")
    _refused(mp, keep(k=None), "null leaf")
    _refused(mp, keep(k=A + 512), "overlap")
    _refused(mp, keep(k=A), "overlap")
    _refused(mp, keep(_cache(mp, n_seqs=1 << 28)), "too many")
    _refused(mp, attend(q=None), "null q")
    _refused(mp, attend(Hq=7), "Hq")
    _refused(mp, attend(Hq=18), "group")
    _refused(mp, attend(window=-1), "window")
    _refused(mp, attend(scale=math.nan), "softmax_scale")
    _refused(mp, attend(out=A), "overlap")
    _refused(mp, attend(size=5), "workspace")
    _refused(mp, attend(ws=None), "workspace")
    assert plan(T=0) == mp.MP_OK and plan(_cache(mp, n_seqs=0)) == mp.MP_OK and keep(_cache(mp, n_seqs=0)) == mp.MP_OK and attend(T=0) == mp.MP_OK


def test_a_missing_mask_or_norm_is_not_the_plain_call(mp):
    for call in (lambda: object.__new__(mp.MpPagedKv).mp_paged_tree_attention(None, None), lambda: object.__new__(mp.MpRotary).mp_norm_rotary(None, None)):
        with pytest.raises(mp.MpError, match="is missing") as e:
            call()
        assert e.value.status == mp.MP_EINVAL
