"""GPU: what the plan of a tree holds in rows without a result: tokens past its masks, and rows of no sequence."""
import pytest
import torch

from tests.paged_util import Batch
from tests.tree_util import ancestors, random_parents, words_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,words,front,back", [
    ([70, 10], 1, 0, 0), ([10, 70], 1, 2, 3), ([200, 0, 1000], 1, 0, 5), ([300], 4, 70, 900), ([130, 129], 2, 1, 0), ([0, 0], 1, 3, 4), ([1100, 3], 16, 0, 1), ([5], 3, 1100, 1100), ([], 2, 0, 9),
])
def test_rows_without_a_result(new, words, front, back):
    from paper_2506_13059_amd import binding as mp
    print(f"case new={new} words={words} front={front} back={back}", flush=True)
    parents = [random_parents(n, 7 * s + 1) for s, n in enumerate(new)]
    if new:
        b = Batch(new, [n + 30 for n in new], 1, 16, pad_front=front, pad_back=back)
        paged, starts, T = b.paged(), b.starts, b.T
    else:
        K = torch.zeros(2, 1, 16, 128, dtype=torch.bfloat16, device="cuda")
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")      # noqa: E731
        paged, starts, T = mp.MpPagedKv(K, K.clone(), i32(0, 4), i32(0), i32(1)), [0], back
    at = torch.tensor([1] * front + sum(parents, []) + [0] * back, dtype=torch.int32, device="cuda")
    want_mask, want_pos, has = [[0] * words for _ in range(T)], [-1] * T, [False] * T
    for s, p in enumerate(parents):
        for i in range(min(new[s], 64 * words)):
            path = ancestors(p, i)
            want_mask[starts[s] + i], want_pos[starts[s] + i], has[starts[s] + i] = words_of(path, words), 30 + len(path) - 1, True
    stale = [torch.full((T, words), 77, dtype=torch.int64, device="cuda"), torch.full((T,), 77, dtype=torch.int32, device="cuda")]
    del stale                                      # (what a tensor that is made next may hold)
    mask, positions = paged.mp_paged_tree_plan(at, words)
    assert mask.tolist() == want_mask and positions.tolist() == want_pos
    # where one is passed, the other is made: each as it is described
    mine = torch.full((T, words), 77, dtype=torch.int64, device="cuda")
    mask, positions = paged.mp_paged_tree_plan(at, words, mask=mine)
    assert mask is mine and mask.tolist() == [m if h else [77] * words for m, h in zip(want_mask, has)] and positions.tolist() == want_pos
    mine = torch.full((T,), 77, dtype=torch.int32, device="cuda")
    mask, positions = paged.mp_paged_tree_plan(at, words, positions=mine)
    assert positions is mine and mask.tolist() == want_mask and positions.tolist() == [p if h else 77 for p, h in zip(want_pos, has)]


def test_words_past_the_limit_are_refused():
    from paper_2506_13059_amd import binding as mp
    b = Batch([3], [20], 1, 16)
    for words in (-1, 0, 17, 256, 257, 272):
        with pytest.raises(mp.MpError) as e:
            b.paged().mp_paged_tree_plan(torch.zeros(3, dtype=torch.int32, device="cuda"), words)
        assert e.value.status == mp.MP_EINVAL
