"""GPU: tensors that the calls over a paged cache make for their results are made by torch's operators, so that modes which look at these see them."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from tests.paged_util import Batch

pytestmark = pytest.mark.gpu


class Made(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.at = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if isinstance(out, torch.Tensor):
            self.at.append((out.data_ptr(), tuple(out.shape), out.dtype))
        return out


def test_results_are_seen_by_dispatch_modes():
    from paper_2506_13059_amd import binding as mp
    b = Batch([5, 3], [40, 30], 2, 16)
    rows = lambda h: torch.randn(8, h, 128, device="cuda").to(torch.bfloat16)      # noqa: E731
    q, k, v = rows(4), rows(2), rows(2)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    pos, parents, leaf = i32(*range(8)), i32(-1, 0, 0, 1, 3, -1, 0, 1), i32(4, 2)
    rot, norm, paged = mp.MpRotary(), mp.MpHeadNorm(torch.ones(128, dtype=torch.bfloat16, device="cuda")), b.paged()
    mask = paged.mp_paged_tree_plan(parents, 1)[0]
    calls = dict(
        rotary=lambda: rot.mp_rotary(q, pos, lookup_position=7), norm=lambda: rot.mp_norm_rotary(norm, q, pos, lookup_position=7),
        append=lambda: paged.mp_paged_append(k, v, rotary=rot, q=q), append_norm=lambda: paged.mp_paged_append_norm(k, v, rotary=rot, q=q, q_norm=norm),
        attention=lambda: paged.mp_paged_attention(q), tree=lambda: paged.mp_paged_tree_attention(q, mask), plan=lambda: paged.mp_paged_tree_plan(parents, 2),
        keep=lambda: paged.mp_paged_tree_keep(mask, leaf), gather=lambda: paged.mp_paged_gather(20),
    )
    for name, call in calls.items():
        with Made() as made:
            got = call()
        for t in got if isinstance(got, tuple) else (got,):
            assert (t.data_ptr(), tuple(t.shape), t.dtype) in made.at, name
            assert t.is_contiguous() and t.device == q.device
