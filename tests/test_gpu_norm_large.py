"""GPU: norms of rows whose squares' sum passes fp32: finite rows are normed as all others are, against the formula in 64 bits."""
import math

import pytest
import torch

from tests.paged_util import Batch, check, gen, turned
from tests.test_gpu_norm_rotary import bound, normed

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.bfloat16).max


def _rows():
    """Rows about the place where the sum of squares passes fp32 (128 elements of 1.6e18), up to the type's largest, and some that have few such elements."""
    x = torch.randn(40, 4, 128, generator=gen(1), device="cuda")
    for t in range(30):
        x[t, 0] = x[t, 0].clamp(-3, 3) * min(10.0 ** (17 + 0.75 * t), LARGEST / 3)
    x[30, 0], x[31, 0] = LARGEST, -LARGEST
    x[32, 0, ::2], x[32, 0, 1::2] = LARGEST, -LARGEST
    x[33, 0, 7] = 3e18
    x[34, 0, 7], x[34, 0, 100] = 1e38, 2.0
    x[35, 0, 127] = LARGEST
    x[36, 0] = 1.6303e18
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("rot,interleaved", [(128, 0), (128, 1), (64, 0), (20, 1)])
@pytest.mark.parametrize("per_head,offset,eps", [(False, 0.0, 1e-6), (True, 1.0, 1e-5), (False, 0.0, 3e38), (False, 64.0, 1e-6)])
def test_large_rows(rot, interleaved, per_head, offset, eps):
    from paper_2506_13059_amd import binding as mp
    x = _rows()
    w = (2.0 + 0.3 * torch.randn(*((4,) if per_head else ()), 128, generator=gen(2), device="cuda")).to(torch.bfloat16)
    norm, spec = mp.MpHeadNorm(w, offset=offset, eps=eps), mp.MpRotary(rot_dim=rot, base=1e4, layout=interleaved, amplitude=1.125)
    pos = torch.arange(40, dtype=torch.int32, device="cuda") * 3001
    out, look = spec.mp_norm_rotary(norm, x, pos, lookup_position=4096)
    xn = normed(x, w, offset, float(torch.tensor(eps)))
    for got, p in ((out, pos), (look, torch.full_like(pos, 4096))):
        want = turned(xn, p, spec.freqs, interleaved, 1.125)
        check(got, want, bound(xn, want, spec.freqs, interleaved, 1.125), "rows")
    b = Batch([40], [50], 4, 16)
    q = b.paged().mp_paged_append_norm(x, x, rotary=spec, q=x, q_norm=norm, k_norm=norm, positions=pos)
    page, slot = b.where(0, b.positions(0))
    assert torch.equal(q, out) and torch.equal(b.K[page, :, slot], out) and torch.equal(b.V[page, :, slot], x)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_the_largest_elements_beside_an_infinity(interleaved):
    from paper_2506_13059_amd import binding as mp
    x = torch.full((4, 2, 128), LARGEST, dtype=torch.bfloat16, device="cuda")
    x[:, 0, 9] = -math.inf
    x[:, 1, 9] = math.nan
    norm, spec = mp.MpHeadNorm(torch.full((128,), 5.0, dtype=torch.bfloat16, device="cuda")), mp.MpRotary(layout=interleaved)
    out = spec.mp_norm_rotary(norm, x, torch.arange(4, dtype=torch.int32, device="cuda") + 5)
    pair = sorted([9, 8 if interleaved else 73])
    assert all(out[t, 0].isnan().nonzero()[:, 0].tolist() == pair for t in range(4)) and (out[:, 0].nan_to_num(0.0) == 0).all()
    assert out[:, 1].isnan().all()
