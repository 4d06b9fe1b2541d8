"""GPU: mp_rotary against the formula in 64 bits."""
import math

import pytest
import torch

from tests.paged_util import check, gen, turn_bound, turned

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


def _x(T, H, seed=1):
    return torch.randn(T, H, 128, generator=gen(seed), device="cuda").to(torch.bfloat16)


def _positions(T, lo=0, hi=200000, seed=2):
    return torch.randint(lo, hi, (T,), generator=gen(seed), device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("rot", [2, 10, 16, 20, 36, 64, 72, 96, 126, 128])
@pytest.mark.parametrize("T,H", [(1, 1), (3, 5), (17, 8)])
def test_layouts_and_parts_of_the_head(T, H, rot, interleaved):
    mp = _mp()
    print(f"case T={T} H={H} rot={rot} interleaved={interleaved}", flush=True)
    r = mp.MpRotary(rot_dim=rot, layout=interleaved, base=1e4, amplitude=1.25)
    x, p = _x(T, H), _positions(T)
    out = r.mp_rotary(x, p)
    want = turned(x, p, r.freqs, interleaved, 1.25)
    check(out, want, turn_bound(x, want, r.freqs, interleaved, 1.25), "rotary")
    assert torch.equal(out[..., rot:], x[..., rot:])


@pytest.mark.parametrize("T,H", [(1, 40), (2, 3), (130, 32), (700, 48), (9001, 7), (40000, 1)])
def test_sizes(T, H):
    mp = _mp()
    print(f"case T={T} H={H}", flush=True)
    r = mp.MpRotary(base=1e6)
    x, p = _x(T, H), _positions(T)
    want = turned(x, p, r.freqs, 0)
    check(r.mp_rotary(x, p), want, turn_bound(x, want, r.freqs, 0), "rotary")


def test_far_and_negative_positions():
    mp = _mp()
    r = mp.MpRotary(base=5e5, layout=mp.MP_ROTARY_INTERLEAVED)
    x = _x(8, 4)
    p = torch.tensor([0, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 1 << 20, -131071, 999999937], dtype=torch.int32, device="cuda")
    want = turned(x, p, r.freqs, 1)
    check(r.mp_rotary(x, p), want, turn_bound(x, want, r.freqs, 1), "rotary")


@pytest.mark.parametrize("H", [1, 8, 33])
def test_rows_of_a_fused_projection_and_the_lookup_position(H):
    mp = _mp()
    r = mp.MpRotary(rot_dim=64, base=1e4)
    fused, p = _x(77, H + 9), _positions(77)
    x = fused[:, 4:4 + H]
    room = torch.full((77, H + 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out, look = r.mp_rotary(x, p, out=room[:, 1:1 + H], lookup_position=4096)
    assert (room[:, 0] == 7).all() and (room[:, -1] == 7).all()
    want = turned(x, p, r.freqs, 0)
    check(out, want, turn_bound(x, want, r.freqs, 0), "out")
    want = turned(x, torch.full_like(p, 4096), r.freqs, 0)
    check(look, want, turn_bound(x, want, r.freqs, 0), "lookup")
    none, alone = r.mp_rotary(x, lookup_position=4096)
    assert none is None and torch.equal(alone, look)
    # in place
    y = x.contiguous()
    got, look2 = r.mp_rotary(y, p, out=y, lookup_position=4096)
    assert got is y and torch.equal(y, out) and torch.equal(look2, look)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_rest_of_the_head_holds_anything(interleaved):
    mp = _mp()
    r = mp.MpRotary(rot_dim=20, layout=interleaved)
    x, p = _x(5, 3), _positions(5)
    x[0, 0, 20], x[1, 1, 21], x[2, 2, 127] = math.inf, -math.inf, math.nan
    out = r.mp_rotary(x, p)
    assert torch.equal(out[..., 20:].nan_to_num(nan=3.0, posinf=4.0, neginf=5.0), x[..., 20:].nan_to_num(nan=3.0, posinf=4.0, neginf=5.0))
    assert out[..., :20].isfinite().all()


@pytest.mark.parametrize("interleaved", [0, 1])
def test_gradient_is_the_rotation_back(interleaved):
    mp = _mp()
    r = mp.MpRotary(rot_dim=96, layout=interleaved, amplitude=0.75)
    x, g, p = _x(6, 3, 5), _x(6, 3, 6), _positions(6)
    leaf = x.double().requires_grad_()
    turned(leaf, p, r.freqs, interleaved, 0.75).backward(g.double())
    got = r.mp_rotary(g, -p)
    check(got, leaf.grad, turn_bound(g, leaf.grad, r.freqs, interleaved, 0.75), "gradient")
    # and against differences of the formula along one direction
    d = torch.randn(x.shape, generator=gen(9), device="cuda", dtype=torch.float64)
    diff = ((turned(x.double() + d, p, r.freqs, interleaved, 0.75) - turned(x.double() - d, p, r.freqs, interleaved, 0.75)) * g.double()).sum() / 2
    assert abs((got.double() * d).sum() - diff) <= (turn_bound(g, leaf.grad, r.freqs, interleaved, 0.75) * d.abs()).sum()


def test_another_stream_and_replays():
    mp = _mp()
    r = mp.MpRotary()
    x, p = _x(32, 8), _positions(32)
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r.mp_rotary(x, p, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            r.mp_rotary(x, p, out=out)
    for i in range(3):
        p.add_(1 + i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, r.mp_rotary(x, p))


def test_refusals():
    mp = _mp()
    r = mp.MpRotary()
    x, p = _x(4, 2), _positions(4)
    for call in (lambda: r.mp_rotary(x.float(), p), lambda: r.mp_rotary(x, p[:3]), lambda: r.mp_rotary(x, p.long()), lambda: r.mp_rotary(x),
                 lambda: r.mp_rotary(x, out=x), lambda: r.mp_rotary(x, p, out_lookup=x), lambda: r.mp_rotary(x.cpu(), p), lambda: r.mp_rotary(x.transpose(0, 1), p[:2]),
                 lambda: r.mp_rotary(x[..., :64], p), lambda: r.mp_rotary(x, p, out=torch.empty(4, 3, 128, dtype=torch.bfloat16, device="cuda")),
                 lambda: mp.MpRotary(rot_dim=64, freqs=r.freqs), lambda: r.mp_rotary(x.view(-1)[4:].view(-1)[:512].view(2, 2, 128), p[:2])):
        with pytest.raises(mp.MpError) as e:
            call()
        assert e.value.status == mp.MP_EINVAL
    assert r.mp_rotary(x[:0], p[:0]).shape == (0, 2, 128)
