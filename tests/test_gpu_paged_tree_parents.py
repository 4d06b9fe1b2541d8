"""GPU: ancestors where parents are numbers far from any token's."""
import pytest
import torch

from tests.paged_util import Batch
from tests.tree_util import ancestors, words_of

pytestmark = pytest.mark.gpu

FAR = [-2 ** 31, -2 ** 31 + 1, -65536, -65535, -65530, -40000, -32769, -32768, -1, 40000, 65536, 2 ** 31 - 1]


@pytest.mark.parametrize("new,words", [([40], 1), ([12, 64, 3], 1), ([130], 3), ([1024, 300], 16)])
def test_parents_that_are_no_token_before_them(new, words):
    from paper_2506_13059_amd import binding as mp  # noqa: F401
    print(f"case new={new} words={words}", flush=True)
    b = Batch(new, [n + 30 for n in new], 1, 16)
    # every second token follows the one before it, and that one no one
    parents = [[FAR[i // 2 % len(FAR)] if i % 2 == 0 else i - 1 for i in range(n)] for n in new]
    mask, positions = b.paged().mp_paged_tree_plan(torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda"), words)
    paths = [ancestors([q if 0 <= q < i else -1 for i, q in enumerate(p)], i) for p in parents for i in range(len(p))]
    assert mask.tolist() == [words_of(p, words) for p in paths]
    assert positions.tolist() == [30 + len(p) - 1 for p in paths]
