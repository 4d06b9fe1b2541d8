"""GPU: norms of each head with the rotation in the same pass, by themselves and on the way into the paged cache, against the formula in 64 bits."""
import pytest
import torch

from tests.paged_util import BF16, Batch, check, gen, turned

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


def _rows(T, H, seed, scale=1.0):
    return (scale * torch.randn(T, H, 128, generator=gen(seed), device="cuda")).to(torch.bfloat16)


def _weight(heads, seed, offset=0.0):
    return (1.0 - offset + 0.3 * torch.randn(*((heads,) if heads else ()), 128, generator=gen(seed), device="cuda")).to(torch.bfloat16)


def normed(x, weight, offset, eps):
    x = x.double()
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) / 128 + eps) * (weight.double() + offset)


def bound(xn, want, freqs, interleaved, amplitude=1.0):
    """One rounding to bf16.  In fp32, in units of 2^-24 of the pair's elements: the sum of squares 12 and its root 6, 1 / sqrt 2, the offset 1, four products and a sum 5, and the
    rotation's 16 (as of rows that are only turned): 30."""
    r = 2 * freqs.numel()
    size = xn.abs()
    pair = size[..., :r]
    pair = pair + (pair.unflatten(-1, (r // 2, 2)).flip(-1).flatten(-2) if interleaved else pair.roll(r // 2, dims=-1))
    size = torch.cat([pair * abs(amplitude), size[..., r:]], dim=-1)
    return BF16 * want.abs() + 2.0 ** -19 * size + 2.0 ** -130


@pytest.mark.parametrize("T,H,rot,interleaved,per_head,offset,eps", [
    (1, 1, 128, 0, False, 0.0, 1e-6), (1, 32, 128, 0, True, 0.0, 1e-6), (16, 8, 64, 1, False, 1.0, 1e-5), (17, 5, 96, 0, True, 1.0, 1e-6),
    (3, 7, 20, 0, False, -0.25, 1e-3), (3, 7, 20, 1, True, 0.0, 1e-6), (2, 3, 2, 0, True, 0.0, 1e-6), (700, 40, 128, 1, True, 0.0, 1e-6), (9001, 3, 128, 0, False, 0.0, 1e-6),
    (8191, 40, 128, 0, True, 1.0, 1e-6),
])
def test_rows(T, H, rot, interleaved, per_head, offset, eps):
    mp = _mp()
    print(f"case T={T} H={H} rot={rot} interleaved={interleaved} per_head={per_head}", flush=True)
    fused = _rows(T, H + 2, 3, 3.0)
    x = fused[:, 1:1 + H]
    x[T // 2, H - 1] = 0                           # a row of zeros stays one
    x[0, 0] *= 2.0 ** -9                           # eps counts here
    spec = mp.MpRotary(rot_dim=rot, base=1e4, layout=interleaved, amplitude=1.125)
    w = _weight(H if per_head else 0, 4, offset)
    norm = mp.MpHeadNorm(w, offset=offset, eps=eps)
    pos = torch.randint(-5, 200000, (T,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    out, look = spec.mp_norm_rotary(norm, x, pos, lookup_position=4096)
    for lo in range(0, T, 1024):
        s = slice(lo, lo + 1024)
        xn = normed(x[s], w, offset, eps)
        for got, p in ((out[s], pos[s]), (look[s], torch.full_like(pos[s], 4096))):
            want = turned(xn, p, spec.freqs, interleaved, 1.125)
            check(got, want, bound(xn, want, spec.freqs, interleaved, 1.125), "rows")
    # each alone, and in place, is the same
    assert torch.equal(spec.mp_norm_rotary(norm, x, pos), out)
    assert torch.equal(spec.mp_norm_rotary(norm, x, lookup_position=4096)[1], look)
    assert spec.mp_norm_rotary(norm, x, pos, out=x) is x and torch.equal(x, out)
    assert (fused[:, 0] == _rows(T, H + 2, 3, 3.0)[:, 0]).all()


def test_rows_that_are_not_finite():
    mp = _mp()
    x = _rows(4, 2, 1)
    x[0, 0, 5], x[1, 1, 7], x[2, 0] = float("inf"), float("nan"), 3e18
    clean = _rows(4, 2, 1)
    spec, norm = mp.MpRotary(rot_dim=64), mp.MpHeadNorm(_weight(0, 2))
    pos = torch.arange(4, dtype=torch.int32, device="cuda") + 1
    got, want = spec.mp_norm_rotary(norm, x, pos), spec.mp_norm_rotary(norm, clean, pos)
    assert got[0, 0].isnan().nonzero()[:, 0].tolist() == [5, 37] and (got[0, 0].nan_to_num(0.0) == 0).all()
    assert got[1, 1].isnan().all()
    for t, h in ((0, 1), (1, 0), (2, 1), (3, 0), (3, 1)):
        assert torch.equal(got[t, h], want[t, h])


@pytest.mark.parametrize("new,lens,Hq,Hkv,page,norms,own_positions,interleaved", [
    ([1], [1], 4, 1, 16, "qk", False, 0),
    ([1] * 16, [5 + 100 * i for i in range(16)], 32, 8, 16, "qk", True, 0),
    ([5, 0, 33, 1], [5, 40, 40, 1], 10, 2, 8, "QK", False, 1),
    ([300, 200], [1000, 200], 5, 5, 64, "Qk", True, 0),
    ([3, 1], [3, 9], 6, 3, 1, "k", False, 1),
    ([7], [9], 3, 1, 32, "q", True, 0),
    ([7], [9], 3, 1, 32, "", True, 1),
    ([4099], [5000], 8, 8, 256, "qK", False, 0),
    ([2, 900], [12, 900], 0, 2, 16, "K", True, 0),
])
def test_append(new, lens, Hq, Hkv, page, norms, own_positions, interleaved):
    """norms: q, k for those with one weight for all heads, Q, K for weights of each head."""
    mp = _mp()
    print(f"case new={new[:6]} lens={lens[:6]} Hq={Hq} Hkv={Hkv} page={page} norms={norms}", flush=True)
    b = Batch(new, lens, Hkv, page, pad_front=2, pad_back=3)
    rot = mp.MpRotary(rot_dim=64, base=1e4, layout=interleaved, amplitude=1.125)
    fused = _rows(b.T, Hq + 2 * Hkv, 5)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    weights = {"q": _weight(Hq if "Q" in norms else 0, 7, 1.0), "k": _weight(Hkv if "K" in norms else 0, 8)}
    q_norm = mp.MpHeadNorm(weights["q"], offset=1.0, eps=1e-5) if "q" in norms.lower() else None
    k_norm = mp.MpHeadNorm(weights["k"], eps=1e-6) if "k" in norms.lower() else None
    place = torch.cat([b.positions(i) for i in range(len(new))])
    turn_to = torch.randint(0, 100000, (b.T,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda() if own_positions else None
    rows = slice(b.starts[0], b.starts[-1])
    position = turn_to[rows] if own_positions else place
    before = b.K.clone(), b.V.clone()
    q_out = torch.full((b.T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda") if Hq else None
    b.paged().mp_paged_append_norm(k, v, rotary=rot, q=q if Hq else None, q_out=q_out, q_norm=q_norm if Hq else None, k_norm=k_norm, positions=turn_to)
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
    page_at, slot = b.table[seq, place // page].long(), place % page
    for x, got, what, offset, eps, there in ((q, q_out, "q", 1.0, 1e-5, q_norm), (k, b.K[page_at, :, slot], "k", 0.0, 1e-6, k_norm)):
        if got is None:
            continue
        if what == "q":
            assert (got[:b.starts[0]] == 7).all() and (got[b.starts[-1]:] == 7).all()
            got = got[rows]
        xn = normed(x[rows], weights[what], offset, eps) if there else x[rows].double()
        want = turned(xn, position, rot.freqs, interleaved, 1.125)
        check(got, want, bound(xn, want, rot.freqs, interleaved, 1.125), what)
    assert torch.equal(b.V[page_at, :, slot], v[rows])
    # nothing else has changed
    b.K[page_at, :, slot], b.V[page_at, :, slot] = before[0][page_at, :, slot], before[1][page_at, :, slot]
    assert torch.equal(b.K.view(torch.int16), before[0].view(torch.int16)) and torch.equal(b.V.view(torch.int16), before[1].view(torch.int16))


def test_append_without_norms_is_that_of_plain_rows():
    mp = _mp()
    b, c = (Batch([5, 40], [30, 40], 3, 16, seed=2) for _ in range(2))
    k, v, q = _rows(45, 3, 1), _rows(45, 3, 2), _rows(45, 6, 3)
    k[3, 1, 100], q[4, 2, 127] = float("inf"), float("nan")            # (dims that are not turned keep every bit)
    rot = mp.MpRotary(rot_dim=64)
    x, y = b.paged().mp_paged_append(k, v, rotary=rot, q=q), c.paged().mp_paged_append_norm(k, v, rotary=rot, q=q)
    assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    x = c.paged().mp_paged_append_norm(k, v, q=q, positions=torch.zeros(45, dtype=torch.int32, device="cuda"))      # no rotation: as they come
    assert torch.equal(x.view(torch.int16), q.view(torch.int16))
    place = torch.cat([b.positions(i) for i in range(2)])
    b.paged().mp_paged_append(k, v, rotary=rot)
    c.paged().mp_paged_append_norm(k, v, rotary=rot, positions=place.int())
    assert torch.equal(b.K.view(torch.int16), c.K.view(torch.int16)) and torch.equal(b.V.view(torch.int16), c.V.view(torch.int16))


def test_norms_without_a_rotation():
    mp = _mp()
    b = Batch([5], [30], 3, 16, seed=2)
    k, v, q = _rows(5, 3, 1), _rows(5, 3, 2), _rows(5, 6, 3)
    w = _weight(6, 1)
    got = b.paged().mp_paged_append_norm(k, v, q=q, q_norm=mp.MpHeadNorm(w))
    want = normed(q, w, 0.0, 1e-6)
    check(got, want, BF16 * want.abs() + 2.0 ** -20 * want.abs(), "q")
    page, slot = b.where(0, b.positions(0))
    assert torch.equal(b.K[page, :, slot], k)


def test_append_drops_what_has_no_place():
    mp = _mp()
    b = Batch([4, 6, 3], [2, 40, 35], 2, 16)          # two of the first sequence's tokens stand before position zero
    b.table[1, 2] = -1                                # keys 32 .. 39 of the second have no page
    b.table[2, 2] = b.n_pages                         # nor have keys 32 .. 34 of the third
    k, v, q = _rows(b.T, 2, 1), _rows(b.T, 2, 2), _rows(b.T, 4, 3)
    before = b.K.clone(), b.V.clone()
    w = mp.MpHeadNorm(_weight(0, 1))
    rot = mp.MpRotary()
    pos = torch.arange(b.T, dtype=torch.int32, device="cuda") + 10
    out = b.paged().mp_paged_append_norm(k, v, rotary=rot, q=q, q_norm=w, k_norm=w, positions=pos)
    assert torch.equal(out, rot.mp_norm_rotary(w, q, pos))
    page, slot = b.where(0, torch.arange(2, device="cuda"))
    assert torch.equal(b.K[page, :, slot], rot.mp_norm_rotary(w, k, pos)[2:4]) and torch.equal(b.V[page, :, slot], v[2:4])
    b.K[page, :, slot], b.V[page, :, slot] = before[0][page, :, slot], before[1][page, :, slot]
    assert torch.equal(b.K.view(torch.int16), before[0].view(torch.int16)) and torch.equal(b.V.view(torch.int16), before[1].view(torch.int16))
