"""GPU: prompts of different lengths in one paged cache become indices of their own, a length at a time, through descriptions of parts of the batch."""
import math

import pytest
import torch

from tests.paged_util import Batch, check, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [8, 64])
def test_sequences_of_different_lengths_become_indices(page):
    from paper_2506_13059_amd import binding as mp
    Hq, Hkv, lens = 8, 2, [700, 431, 700]
    b = Batch([1, 1, 1], lens, Hkv, page)
    q = torch.randn(3, Hq, 128, generator=gen(3), device="cuda").to(torch.bfloat16)
    whole = b.paged().mp_paged_attention(q, max_new=1)
    want, _, _, _ = b.attention(q)
    all_k, all_v = b.paged().mp_paged_gather(max(lens))
    assert (all_k[1, :, 431:] == 0).all() and (all_v[1, :, 431:] == 0).all()           # (not for an index: they would be keys)
    for i, n in enumerate(lens):
        part = mp.MpPagedKv(b.K, b.V, b.table[i:i + 1], b.kv_len[i:i + 1], b.q_start[i:i + 2])
        k, v = part.mp_paged_gather(n)
        assert torch.equal(k[0], b.keys[i]) and torch.equal(v[0], b.values[i]) and torch.equal(k[0], all_k[i, :, :n])
        ctx = mp.MpContext(1, Hq, Hkv, max_tokens=n, levels=1, max_fine=64)
        ctx.mp_cluster_kv(k, v, 40, iters=3)
        out = ctx.mp_decode_attention(q[i:i + 1], key_budget=n)                         # (a budget for all keys: attention itself)
        K, V = b.keys[i].double().repeat_interleave(4, dim=0), b.values[i].double().repeat_interleave(4, dim=0)
        w = torch.softmax((K @ q[i].double()[:, :, None])[..., 0] / math.sqrt(128), dim=1)
        size = (w[:, :, None] * V.abs()).sum(1)
        bound = 2.0 ** -8 * want[i].abs() + 2.0 ** -8 * size                            # one rounding of the result, one of the weights
        check(out[0], want[i], bound, f"index of sequence {i}")
        check(whole[i], want[i], bound, f"pages of sequence {i}")
        ctx.close()
