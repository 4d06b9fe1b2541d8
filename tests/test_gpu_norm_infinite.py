"""GPU: norms of rows with an infinity: NaN in that element and in its partner of the rotation, if it has one, and zero elsewhere."""
import math

import pytest
import torch

from tests.paged_util import Batch, gen

pytestmark = pytest.mark.gpu


def _partner(d, rot, interleaved):
    return d if d >= rot else d ^ 1 if interleaved else (d + rot // 2) % rot


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("rot", [2, 20, 64, 96, 126, 128])
@pytest.mark.parametrize("per_head", [False, True])
def test_an_infinity_stays_with_its_pair(rot, interleaved, per_head):
    from paper_2506_13059_amd import binding as mp
    T = 128                                        # token t: the infinity in dim t of its second head
    x = torch.randn(T, 3, 128, generator=gen(1), device="cuda").to(torch.bfloat16)
    clean = x.clone()
    x[torch.arange(T), 1, torch.arange(T)] = math.inf
    x[::2, 1] *= -1.0
    w = (1 + 0.3 * torch.randn(*((3,) if per_head else ()), 128, generator=gen(2), device="cuda")).to(torch.bfloat16)
    norm, spec = mp.MpHeadNorm(w), mp.MpRotary(rot_dim=rot, base=1e4, layout=interleaved)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 1
    want = torch.zeros(T, 128, dtype=torch.bool)
    for t in range(T):
        want[t, [t, _partner(t, rot, interleaved)]] = True

    def as_promised(got, plain):
        assert torch.equal(got[:, 1].isnan().cpu(), want) and (got[:, 1].nan_to_num(0.0) == 0).all()
        assert torch.equal(got[:, ::2], plain[:, ::2])
    out, look = spec.mp_norm_rotary(norm, x, pos, lookup_position=77)
    out1, look1 = spec.mp_norm_rotary(norm, clean, pos, lookup_position=77)
    as_promised(out, out1)
    as_promised(look, look1)
    # on the way into the cache
    b = Batch([T], [T], 3, 16)
    q = b.paged().mp_paged_append_norm(x, clean, rotary=spec, q=x, q_norm=norm, k_norm=norm, positions=pos)
    page, slot = b.where(0, b.positions(0))
    as_promised(q, out1)
    as_promised(b.K[page, :, slot], out1)
