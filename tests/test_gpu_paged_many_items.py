"""GPU: attention of 33 to 128 query rows a KV head in batches of 128 and more sequences times KV heads, whose parts are put together by kernels for many items: few parts a cut and, of a long
sequence among short ones, more than four and more than 32."""
import math

import pytest
import torch

from tests.paged_util import Batch, check, gen
from tests.test_gpu_paged_tree import _attend, _trees

pytestmark = pytest.mark.gpu

BATCHES = [
    # new tokens, keys behind them, KV heads
    ([9, 12, 16], [700, 41, 1500], 32, 43),                          # shares that end within most items
    ([16, 1, 0, 12], [900, 3, 60, 300], 4, 36),
    ([12] + [1, 9, 16], [30000] + [5, 0, 17], 2, 64),                # (the first one's parts: more than 32)
    ([16, 10], [5000, 40], 16, 8),
    ([11], [0], 1, 200),                                             # new tokens alone
]


def _batch(new, older, Hkv, seqs, page, **kw):
    n = [new[0]] + [new[1 + i % (len(new) - 1)] if len(new) > 1 else new[0] for i in range(seqs - 1)]
    k = [older[0]] + [older[1 + i % (len(older) - 1)] if len(older) > 1 else older[0] for i in range(seqs - 1)]
    b = Batch(n, [x + y for x, y in zip(n, k)], Hkv, page, pad_front=1, pad_back=2, **kw)
    assert seqs * Hkv >= 128
    return b


def _causal(b, G, window=0):
    q = (2.0 * torch.randn(b.T, G * b.Hkv, 128, generator=gen(11), device="cuda")).to(torch.bfloat16)
    out = torch.full((b.T, G * b.Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, G * b.Hkv), 7.0, dtype=torch.float32, device="cuda")
    b.paged().mp_paged_attention(q, max_new=max(b.new), window=window, out=out, lse=lse)
    want, wlse, ob, lb = b.attention(q, window)
    rows = slice(b.starts[0], b.starts[-1])
    assert (out[:b.starts[0]] == 7).all() and (out[b.starts[-1]:] == 7).all() and (lse[:b.starts[0]] == 7).all() and (lse[b.starts[-1]:] == 7).all()
    check(lse[rows], wlse[rows], lb[rows], "lse")
    check(out[rows], want[rows], ob[rows], "out")
    return q, out, lse


@pytest.mark.parametrize("new,older,Hkv,seqs", BATCHES)
@pytest.mark.parametrize("page,window", [(16, 0), (64, 100)])
def test_causal(new, older, Hkv, seqs, page, window):
    """33 to 64 rows: groups of four (of 16 tokens: 64 rows) and of three."""
    for G in (4, 3) if Hkv <= 4 else (4,):
        if not 32 < max(new) * G <= 64:
            continue
        print(f"case new={new} older={older} Hkv={Hkv} seqs={seqs} page={page} window={window} G={G}", flush=True)
        b = _batch(new, older, Hkv, seqs, page)
        b.table[1, 0] = -1
        _causal(b, G, window)


@pytest.mark.parametrize("new,older,Hkv,seqs", BATCHES)
@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("page,window", [(16, 0), (64, 100), (4, 0)])
def test_trees(new, older, Hkv, seqs, G, page, window):
    """33 to 64 rows a KV head, and 65 to 128."""
    print(f"case new={new} older={older} Hkv={Hkv} seqs={seqs} page={page} window={window} G={G}", flush=True)
    if Hkv * G > 64:
        G = 5 if G == 8 else G
    assert 32 < max(new) * G <= 128
    b = _batch(new, older, Hkv, seqs, page)
    b.table[1, 0] = -1
    _attend(b, G * Hkv, _trees(b.new), 1, window)


@pytest.mark.parametrize("G", [4, 8])
def test_a_nan_reaches_the_rows_that_see_it_and_no_others(G):
    """A key of NaN in one sequence: its rows are NaN; what a table's missing pages leave without a key stays zero."""
    b = _batch([12, 12], [9000, 300], 2, 64, 16)
    b.table[2] = -1
    b.keys[0][0, 4000, 5] = math.nan
    page, slot = b.where(0, torch.tensor(4000, device="cuda"))
    b.K[page, 0, slot, 5] = math.nan
    q = torch.randn(b.T, 2 * G, 128, generator=gen(3), device="cuda").to(torch.bfloat16)
    mask = torch.tensor([[(1 << (i + 1)) - 1] for i in range(12)] * 64, dtype=torch.int64, device="cuda")
    mask = torch.cat([torch.zeros_like(mask[:1]), mask, torch.zeros_like(mask[:2])])
    lse = torch.empty(b.T, 2 * G, device="cuda")
    calls = [lambda: b.paged().mp_paged_tree_attention(q, mask, max_new=12, lse=lse)]
    if G == 4:
        calls.append(lambda: b.paged().mp_paged_attention(q, max_new=12, lse=lse))
    for call in calls:
        out = call()
        first, third = slice(b.starts[0], b.starts[1]), slice(b.starts[2], b.starts[3])
        assert out[first, :G].isnan().all() and lse[first, :G].isnan().all()
        assert out[first, G:].isfinite().all() and lse[first, G:].isfinite().all()
        assert (out[third] == 0).all() and (lse[third] == -math.inf).all()
        rest = torch.cat([out[b.starts[1]:b.starts[2]], out[b.starts[3]:b.starts[-1]]])
        assert rest.isfinite().all() and (rest != 0).any(-1).all()


def test_repeated_calls_give_the_same_bits():
    b = _batch([16, 9], [4000, 250], 8, 20, 16)
    q, out, lse = _causal(b, 4)
    lse2 = torch.empty_like(lse)
    for _ in range(3):
        out2 = b.paged().mp_paged_attention(q, max_new=16, lse=lse2)
        rows = slice(b.starts[0], b.starts[-1])
        assert torch.equal(out[rows], out2[rows]) and torch.equal(lse[rows], lse2[rows])
