"""GPU: attention over the paged cache where attended keys or queries are not finite: NaN reaches the rows that it belongs to, in their results and denominators,
and no others."""
import math

import pytest
import torch

from tests.paged_util import BF16, Batch, check, gen

pytestmark = pytest.mark.gpu

# one workgroup finishes the item; parts of several are put together; 16, 32 and 64 rows; chunks, whole and in parts; short ones beside long ones
CASES = [([1], [100], 4), ([1], [5000], 4), ([4], [900], 4), ([5], [700], 6), ([8], [3000], 8), ([80], [80], 4), ([300], [5000], 4), ([100, 1, 30], [700, 300, 900], 2)]


def _clean(new, lens, G, scale=1.0):
    b = Batch(new, lens, 2, 16, pad_front=1, pad_back=1, scale=scale)
    q = (2.0 * torch.randn(b.T, 2 * G, 128, generator=gen(5), device="cuda")).to(torch.bfloat16)
    return b, q


def _attend(b, q, window=0):
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = b.paged().mp_paged_attention(q, max_new=max(b.new), window=window, lse=lse, out=torch.full_like(q, 7.0))
    return out, lse


def _compare(got, want, nan_rows):
    """nan_rows [tokens, heads]: those are NaN throughout; the others are within their bounds of the clean batch's."""
    (out, lse), (wout, wlse, ob, lb) = got, want
    assert out[nan_rows].isnan().all() and lse[nan_rows].isnan().all()
    rest = ~nan_rows & ~wlse.isnan()
    check(out[rest], wout[rest], ob[rest], "out")
    check(lse[rest], wlse[rest], lb[rest], "lse")
    assert (out[wlse.isnan()] == 7).all() and (lse[wlse.isnan()] == 7).all()


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("new,lens,G", CASES)
def test_keys_that_are_nan(new, lens, G, window):
    print(f"case new={new} lens={lens} G={G} window={window}", flush=True)
    b, q = _clean(new, lens, G)
    want = b.attention(q, window)
    n = lens[0]
    for at in (n - 1, max(0, n - new[0] - 1), n - new[0] // 2 - 1, n // 3):
        saved = b.keys[0][1, at].clone()
        b.keys[0][1, at, 77] = math.nan
        b.write()
        hit = torch.zeros(b.T, 2 * G, dtype=torch.bool, device="cuda")
        p = b.positions(0)
        sees = (p >= at) & ((p - at < window) if window else torch.ones_like(p, dtype=torch.bool))
        hit[b.starts[0]:b.starts[1], G:] = sees[:, None]
        _compare(_attend(b, q, window), want, hit)
        b.keys[0][1, at] = saved
        b.write()


@pytest.mark.parametrize("new,lens,G", CASES)
def test_queries_that_are_nan_or_infinite(new, lens, G):
    b, q = _clean(new, lens, G)
    want = b.attention(q)
    hit = torch.zeros(b.T, 2 * G, dtype=torch.bool, device="cuda")
    for token, head, value in ((b.starts[0], 0, math.nan), (b.starts[1] - 1, 2 * G - 1, math.nan), (b.starts[0] + new[0] // 2, G, math.inf)):
        q[token, head, 100] = value                 # (an infinite one: logits of both infinities and, where its key element is zero, NaN)
        hit[token, head] = True
    _compare(_attend(b, q), want, hit)


@pytest.mark.parametrize("new,lens,G", CASES)
def test_logits_that_overflow(new, lens, G):
    """A logit of +inf is a NaN row; one of -inf weighs nothing."""
    b, q = _clean(new, lens, G)
    at = (lens[0] - new[0]) // 2
    b.keys[0][0, :, 7] = 0
    b.keys[0][0, at, 7] = 3e38
    b.write()
    q[..., 7] = 0
    token = b.starts[1] - 1
    q[token, 0] = 0
    out, _, ob, _ = want = b.attention(q)
    q[token, 0, 7] = 3e38
    hit = torch.zeros(b.T, 2 * G, dtype=torch.bool, device="cuda")
    hit[token, 0] = True
    _compare(_attend(b, q), want, hit)
    q[token, 0, 7] = -3e38
    got, lse = _attend(b, q)
    v = b.values[0][0].double()
    others = torch.arange(lens[0], device="cuda") != at
    n = lens[0] - 1
    mean, size = v[others].mean(0), v[others].abs().mean(0)
    check(got[token, 0], mean, BF16 * mean.abs() + (BF16 + (n + 64) * 2.0 ** -24) * size, "row of the others' mean")
    assert abs(lse[token, 0].item() - math.log(n)) <= (n + 64) * 2.0 ** -24 + 2.0 ** -22 * math.log(n)
    rest = ~hit & ~want[1].isnan()
    check(got[rest], out[rest], ob[rest], "out")


@pytest.mark.parametrize("new,G", [(1, 4), (40, 4)])
def test_a_row_of_logits_of_minus_infinity_is_as_one_without_a_key(new, G):
    b, q = _clean([new], [new], G)
    b.keys[0][0, :, 7] = 0
    b.keys[0][0, 0, 7] = 3e38
    b.write()
    q[b.starts[0], :G, 7] = -3e38                   # (the first token attends key 0 alone)
    out, lse = _attend(b, q)
    assert (out[b.starts[0], :G] == 0).all() and (lse[b.starts[0], :G] == -math.inf).all()
    assert out[b.starts[0], G:].isfinite().all()
