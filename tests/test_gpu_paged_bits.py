"""GPU: what append and rotary positions leave as it is, they leave bit for bit, every bf16 pattern among it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _every_pattern():
    return torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(256, 2, 128)


def test_rows_stored_without_a_rotation_keep_every_bit():
    from paper_2506_13059_amd import binding as mp
    x = _every_pattern()
    K, V = (torch.zeros(16, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 16)
    cache = mp.MpPagedKv(K, V, table, *(torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([256], [0, 256])))
    rows = x.view(torch.bfloat16)
    out = cache.mp_paged_append(rows, rows, q=rows)
    assert torch.equal(out.view(torch.int16), x)
    for pages in (V, K):
        assert torch.equal(pages.view(torch.int16).transpose(1, 2).reshape(256, 2, 128), x)


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("rot", [2, 20, 64, 126])
def test_dimensions_that_are_not_turned_keep_every_bit(rot, interleaved):
    from paper_2506_13059_amd import binding as mp
    r = mp.MpRotary(rot_dim=rot, layout=interleaved)
    x = torch.cat([_every_pattern(), _every_pattern().roll(rot, dims=-1)], dim=1)
    out, look = r.mp_rotary(x.view(torch.bfloat16), torch.arange(256, dtype=torch.int32, device="cuda"), lookup_position=9)
    assert torch.equal(out.view(torch.int16)[..., rot:], x[..., rot:]) and torch.equal(look.view(torch.int16)[..., rot:], x[..., rot:])
    K, V = (x[:, :2].transpose(0, 1)[None].clone(memory_format=torch.contiguous_format).view(torch.bfloat16) for _ in range(2))
    cache = mp.MpPagedKv(K, V, *(torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([[0]], [256], [0, 0])))
    k, v, k_lookup = (t.view(torch.int16)[0] for t in cache.mp_paged_gather(256, rotary=r, lookup_position=9))
    want = x[:, :2].transpose(0, 1)
    assert torch.equal(k, want) and torch.equal(v, want) and torch.equal(k_lookup[..., rot:], want[..., rot:])
