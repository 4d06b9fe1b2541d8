"""GPU: the paged cache at the far end of the longest page table that it may have (2^31 - 64 keys a sequence), all of whose keys but the last few are out of sight."""
import math

import pytest
import torch

from tests.paged_util import BF16, check, gen

pytestmark = pytest.mark.gpu

PAGE, HELD = 64, 8                         # rows of a page, pages at the end of the sequence that are there
ENTRIES = 2 ** 31 // PAGE - 1


@pytest.fixture(scope="module")
def table():
    t = torch.full((1, ENTRIES), -1, dtype=torch.int32, device="cuda")
    t[0, -HELD:] = torch.randperm(HELD, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    return t


@pytest.mark.parametrize("behind", [0, 1, 37, 97])
@pytest.mark.parametrize("new,G", [(1, 4), (3, 8), (8, 8), (80, 4)])
def test_last_keys_of_the_longest_table(table, new, G, behind):
    from paper_2506_13059_amd import binding as mp
    Hkv, window = 2, 100
    n = ENTRIES * PAGE - behind                                     # keys; n - first of them are made
    first = n - new - window
    print(f"case new={new} G={G} keys={n}", flush=True)
    g = gen(new + behind)
    k, v = (torch.randn(n - first, Hkv, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(new, G * Hkv, 128, generator=g, device="cuda").to(torch.bfloat16)
    K, V = (torch.full((HELD, Hkv, PAGE, 128), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv_len = torch.tensor([n], dtype=torch.int32, device="cuda")
    mp.MpPagedKv(K, V, table, kv_len, torch.tensor([0, n - first], dtype=torch.int32, device="cuda")).mp_paged_append(k, v)
    paged = mp.MpPagedKv(K, V, table, kv_len, torch.tensor([0, new], dtype=torch.int32, device="cuda"))
    gk, gv = paged.mp_paged_gather(n - first, first=first)
    assert torch.equal(gk[0], k.transpose(0, 1)) and torch.equal(gv[0], v.transpose(0, 1))
    out = paged.mp_paged_attention(q, max_new=new, window=window)
    torch.cuda.synchronize()
    p, j = torch.arange(n - new, n, device="cuda")[:, None], torch.arange(first, n, device="cuda")[None]
    seen = (j <= p) & (p - j < window)
    for h in range(G * Hkv):
        keys, values = k[:, h // G].double(), v[:, h // G].double()
        w = torch.softmax((q[:, h].double() @ keys.t().contiguous() / math.sqrt(128)).masked_fill(~seen, -math.inf), dim=1)
        want, size = w @ values, w @ values.abs()
        # one rounding of the result and one of the probabilities; logits: 130 roundings to fp32 of the products' sum
        d = 130 * 2.0 ** -24 / math.sqrt(128) * q[:, h].double().norm(dim=1, keepdim=True) * keys.norm(dim=1).max()
        check(out[:, h], want, BF16 * want.abs() + (BF16 + 2 * d + (window + 64) * 2.0 ** -24) * size, f"head {h}")
