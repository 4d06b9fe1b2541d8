"""GPU: trees of 33 to 128 query rows a KV head over many blocks of small pages, some of them missing: entries are asked for five blocks ahead."""
import pytest
import torch

from tests.paged_util import Batch
from tests.test_gpu_paged_tree import _attend, _trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,G", [([12], 4), ([16, 9, 16], 4), ([24], 4), ([17, 30, 1, 30], 4), ([128], 1)])
@pytest.mark.parametrize("page", [1, 2, 4, 8])
@pytest.mark.parametrize("context,window", [(64, 0), (250, 0), (321, 130), (9000, 0), (9000, 4000)])
def test_blocks_of_small_pages(new, G, page, context, window):
    print(f"case new={new} G={G} page={page} context={context} window={window}", flush=True)
    lens = [n + context // (1 + 3 * (i % 2)) for i, n in enumerate(new)]
    b = Batch(new, lens, 2, page, pad_front=1, pad_back=1)
    gone = torch.rand(b.table.shape, generator=torch.Generator().manual_seed(page)) < 0.05
    b.table[gone.cuda()] = -1
    _attend(b, 2 * G, _trees(new), -(-max(new) // 64), window)
