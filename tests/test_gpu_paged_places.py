"""GPU: append to the paged cache where tokens stand behind their sequence's page table, at its edges and before its beginning: what is stored, and nothing else."""
import pytest
import torch

from tests.paged_util import Batch, gen

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int16)


@pytest.mark.parametrize("page", [1, 16, 1024])
@pytest.mark.parametrize("behind", [0, 1, 2, 5, 6, 17, 10000, 2 ** 30])
def test_tokens_behind_the_table_are_dropped(page, behind):
    """The second of three sequences ends `behind` keys past the last row that its page table has room for."""
    print(f"case page={page} behind={behind}", flush=True)
    n = 2 * page + 3
    b = Batch([4, 6, 3], [max(n, 4), n, n], 2, page, spare=4)
    entries = b.table.shape[1]
    spare = sorted(set(range(b.n_pages)) - set(b.table[b.table >= 0][b.table[b.table >= 0] < b.n_pages].tolist()))
    b.table[1, -1] = spare[0]                                      # (its last entry names a page of its own)
    room = entries * page
    b.lens[1] = room + behind
    b.kv_len.copy_(torch.tensor(b.lens, dtype=torch.int32))
    k, v, q = (torch.randn(b.T, h, 128, generator=gen(h), device="cuda").to(torch.bfloat16) for h in (2, 2, 6))
    v = v + 1
    want = b.K.clone(), b.V.clone()
    for i in range(3):
        p = b.positions(i)
        for token, at in zip(range(b.starts[i], b.starts[i + 1]), p.tolist()):
            page_at = int(b.table[i, at // page]) if 0 <= at < room else -1
            if 0 <= page_at < b.n_pages:
                want[0][page_at, :, at % page], want[1][page_at, :, at % page] = k[token], v[token]
    out = b.paged().mp_paged_append(k, v, q=q)
    assert torch.equal(_bits(b.K), _bits(want[0])) and torch.equal(_bits(b.V), _bits(want[1])) and torch.equal(out, q)
    if behind >= 6:
        assert (b.positions(1) >= room).all()


def test_rows_of_other_sequences_are_stored_beside_one_without_room():
    """Nothing of a sequence that lies behind its table is stored, wherever its rows come from; the others' are, once each."""
    b = Batch([4, 6, 3], [2, 40, 35], 2, 16)
    b.kv_len[1] = 10000
    k, v = (torch.randn(b.T, 2, 128, generator=gen(i), device="cuda").to(torch.bfloat16) for i in (1, 2))
    want = b.K.clone(), b.V.clone()
    for i, keep in ((0, 2), (2, 3)):                               # (two of the first sequence's tokens stand before position zero)
        at = b.positions(i)[-keep:]
        page, slot = b.where(i, at)
        rows = slice(b.starts[i + 1] - keep, b.starts[i + 1])
        want[0][page, :, slot], want[1][page, :, slot] = k[rows], v[rows]
    b.paged().mp_paged_append(k, v)
    assert torch.equal(_bits(b.K), _bits(want[0])) and torch.equal(_bits(b.V), _bits(want[1]))
