"""GPU: attention over the paged cache holds probabilities in two bf16 parts (2^-15) where it says so.  Values are such that their weighted sum cancels, so that
the rounding of the result does not hide what is left of the probabilities; the same probabilities rounded to bf16 once are shown to miss the bounds."""
import math

import pytest
import torch

from tests.paged_util import BF16, Batch, check, gen

pytestmark = pytest.mark.gpu

SCALE = 1.0 / math.sqrt(128)


def _batch(new, lens, page=16, columns=0):
    """Every third key has a logit 7.8125 / sqrt(128) above the others, of whom one weighs e^-0.6905 = (1 + 0.335 / 128) / 2 then: a third of a step of bf16
    from the next number.  Values are +v of the former, -v of the latter, so that their sums all but cancel."""
    b = Batch(new, lens, 2, page, columns=columns)
    for i, n in enumerate(lens):
        g = gen(40 + i)
        top = (torch.arange(n, device="cuda") % 3 == 0)[None, :, None]
        common = (0.25 * torch.randn(2, 1, 128, generator=g, device="cuda")).to(torch.bfloat16).expand(2, n, 128).clone()
        common[..., 0] = torch.where(top[..., 0], 3.90625, 0.0)
        v = (0.5 + 1.5 * torch.rand(2, 1, 128, generator=g, device="cuda")).to(torch.bfloat16)
        b.keys[i], b.values[i] = common, torch.where(top, v, -v)
    b.write()
    return b


def _bounds(b, i, q):
    """Sequence i's rows in 64 bits, on the CPU: results [tokens, heads, 128], their bounds, and the results with probabilities rounded to bf16 once."""
    G = q.shape[1] // 2
    rows = slice(b.starts[i], b.starts[i + 1])
    n = b.lens[i]
    seen = torch.arange(n)[None] <= torch.arange(n - b.new[i], n)[:, None]
    want, bound, rounded = [], [], []
    for h in range(2 * G):
        k, v, x = b.keys[i][h // G].cpu().double(), b.values[i][h // G].cpu().double(), q[rows, h].cpu().double()
        s = (x @ k.t() * SCALE).masked_fill(~seen, -math.inf)
        e = torch.exp(s - s.amax(1, keepdim=True))
        l = e.sum(1, keepdim=True)
        o, size = e @ v / l, e @ v.abs() / l
        d = 130 * 2.0 ** -24 * SCALE * x.norm(dim=1, keepdim=True) * k.norm(dim=1).max()          # of a logit; sums of n terms in fp32 below
        want.append(o)
        bound.append(BF16 * o.abs() + (2.0 ** -15 + 2 * d + (seen.sum(1, keepdim=True) + 64) * 2.0 ** -24) * size)
        rounded.append(e.to(torch.bfloat16).double() @ v / l)
    return torch.stack(want, 1), torch.stack(bound, 1), torch.stack(rounded, 1)


def _check(b, G, sequences):
    q = torch.randn(b.T, 2 * G, 128, generator=gen(9), device="cuda").to(torch.bfloat16)
    q[..., 0] = 2.0
    out = b.paged().mp_paged_attention(q, max_new=max(b.new)).cpu()
    for i in sequences:
        want, bound, rounded = _bounds(b, i, q)
        assert ((rounded - want).abs() > bound).any(-1).all()           # (one rounding would be seen, in every row)
        check(out[b.starts[i]:b.starts[i + 1]], want, bound, f"sequence {i}")


@pytest.mark.parametrize("page", [16, 4])
@pytest.mark.parametrize("new,lens,G", [([1], [100], 4), ([1], [3000], 4), ([1], [128], 8), ([2], [1111], 8), ([4], [900], 4), ([8], [2000], 4), ([5], [700], 6),
                                        ([4], [2500], 8), ([1] * 20, [90 + 131 * i for i in range(20)], 2), ([1, 3, 2], [300, 200, 3000], 5)])
def test_up_to_32_rows_a_head(new, lens, G, page):
    print(f"case new={new[:4]} lens={lens[:4]} G={G} page={page}", flush=True)
    _check(_batch(new, lens, page), G, range(len(new)))


@pytest.mark.parametrize("G", [1, 4, 8])
def test_short_sequences_beside_long_ones_where_the_table_has_room(G):
    """Up to 16 rows a head beside 90 tokens, in a table with room for 128K keys of each of six sequences, 2 KV heads."""
    new = [1, 2, 1, 90, 1, 2]
    _check(_batch(new, [100, 300, 2999, 400, 129, 1500], columns=8192), G, [i for i, n in enumerate(new) if n * G <= 16])
