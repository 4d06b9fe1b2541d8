"""GPU: trees of drafted tokens, norms and page pools where sizes, streams and arguments could go wrong."""
import math

import pytest
import torch

from tests.paged_util import Batch, check, gen, turned
from tests.test_gpu_norm_rotary import bound as rows_bound
from tests.test_gpu_norm_rotary import normed
from tests.test_gpu_paged_tree import _attend, _mask, _rows, _trees
from tests.tree_util import tree_attention

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


@pytest.mark.parametrize("new,G", [(3, 4), (7, 4), (12, 4), (16, 4), (20, 5), (25, 5), (40, 5)])
@pytest.mark.parametrize("page", [1, 2, 4, 8])
def test_small_pages(new, G, page):
    b = Batch([new, 1, new], [new + 333, 70, new], 2, page, pad_front=1)
    b.table[0, 5] = -1
    _attend(b, 2 * G, _trees(b.new), -(-new // 64), window=0)
    _attend(b, 2 * G, _trees(b.new), -(-new // 64), window=100)


@pytest.mark.parametrize("new,G", [(4, 4), (8, 4), (12, 4), (30, 4), (63, 4)])
def test_caches_past_4_gib(new, G):
    """Pages whose bytes lie past 32 bits in keys and in values: appended to, attended, moved."""
    mp = _mp()
    Hkv, page, n_pages = 4, 64, 83000                        # 5.4 GB each
    free, _ = torch.cuda.mem_get_info()
    if free < 14 << 30:
        pytest.skip("too little memory")
    b = Batch([new], [new + 300], Hkv, page)
    used = b.table[0, :-(-(new + 300) // page)].clone()
    far = (n_pages - 1 - torch.arange(used.numel(), device="cuda") * 3).int()
    K, V = (torch.empty(n_pages, Hkv, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[far.long()], V[far.long()] = b.K[used.long()], b.V[used.long()]
    table = torch.full_like(b.table, -1)
    table[0, :used.numel()] = far
    cache = mp.MpPagedKv(K, V, table, b.kv_len, b.q_start)
    q = _rows(new, G * Hkv, 3)
    marked = _trees([new])
    out = cache.mp_paged_tree_attention(q, _mask(b, marked, 1), max_new=new)
    want, _, ob, _ = tree_attention(b, q, marked)
    check(out, want, ob, "out")
    # the same rows appended again, normed and turned
    rot, norm = mp.MpRotary(base=1e4), mp.MpHeadNorm((1 + 0.2 * torch.randn(Hkv, 128, generator=gen(1), device="cuda")).to(torch.bfloat16))
    k, v = _rows(new, Hkv, 5), _rows(new, Hkv, 6)
    pos = torch.arange(new, dtype=torch.int32, device="cuda") + 7
    cache.mp_paged_append_norm(k, v, rotary=rot, k_norm=norm, positions=pos)
    place = b.positions(0)
    at, slot = table[0].long()[place // page], place % page
    xn = normed(k, norm.weight, 0.0, 1e-6)
    want = turned(xn, pos, rot.freqs, 0)
    check(K[at, :, slot], want, rows_bound(xn, want, rot.freqs, 0), "keys")
    assert torch.equal(V[at, :, slot], v)
    kept = K[at, :, slot].clone()
    path = marked[0][new - 1]
    keep = cache.mp_paged_tree_keep(_mask(b, marked, 1), torch.tensor([new - 1], dtype=torch.int32, device="cuda"))
    assert keep.tolist() == [300 + len(path)]
    assert torch.equal(K[at, :, slot][:len(path)], kept[path]) and torch.equal(V[at, :, slot][:len(path)], v[path])


def test_calls_on_two_streams():
    """Attention of two batches at once, each with a workspace of its own, and page tables of a third beside them."""
    mp = _mp()
    a, b = Batch([12, 5], [3000, 700], 4, 16, seed=1), Batch([30, 63], [2500, 900], 4, 64, seed=2)
    calls = []
    for c in (a, b):
        q, mask = _rows(c.T, 16, 3), _mask(c, _trees(c.new), 1)
        ws = torch.empty(mp.mp_paged_workspace_bytes(c.T, 16, 4, 2, max(c.new)), dtype=torch.uint8, device="cuda")
        calls.append((c.paged(), q, mask, max(c.new), ws, c.paged().mp_paged_tree_attention(q, mask, max_new=max(c.new))))
    table, stack = torch.full((40, 8), -1, dtype=torch.int32, device="cuda"), torch.arange(200, dtype=torch.int32, device="cuda")
    kv_len, q_start, n_free = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (40, 41, 1))
    n_free.fill_(200)
    pool = mp.MpPagePool(table, kv_len, q_start, stack, n_free, 16)
    come = torch.full((40,), 3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[], []]
    for _ in range(20):
        for i, (paged, q, mask, n, ws, _) in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                outs[i].append(paged.mp_paged_tree_attention(q, mask, max_new=n, workspace=ws))
        with torch.cuda.stream(streams[2]):
            pool.mp_paged_reserve(come)
    torch.cuda.synchronize()
    for i, (*_, want) in enumerate(calls):
        assert all(torch.equal(o, want) for o in outs[i])
    assert kv_len.tolist() == [60] * 40 and int(n_free) == 200 - 40 * 4
    held = table[:, :4].flatten()
    assert held.unique().numel() == 160 and (table[:, 4:] == -1).all()


def test_captured_calls_follow_what_their_inputs_hold():
    """Plan, append, attention and keep of a step recorded once, replayed over other trees, lengths and rows, against calls made directly."""
    mp = _mp()
    b = Batch([20, 9, 33], [400, 60, 900], 2, 16, seed=4, pad_back=3)
    rot, norm = mp.MpRotary(), mp.MpHeadNorm(torch.ones(128, dtype=torch.bfloat16, device="cuda"))
    paged = b.paged()
    fused = _rows(b.T, 8 + 4, 1)
    parents, leaf = torch.zeros(b.T, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(mp.mp_paged_workspace_bytes(b.T, 8, 2, 3, 33), dtype=torch.uint8, device="cuda")

    def step():
        mask, positions = paged.mp_paged_tree_plan(parents, 1)
        q = paged.mp_paged_append_norm(fused[:, 8:10], fused[:, 10:], rotary=rot, q=fused[:, :8], q_norm=norm, k_norm=norm, positions=positions)
        out = paged.mp_paged_tree_attention(q, mask, max_new=33, workspace=ws)
        return mask, positions, q, out, paged.mp_paged_tree_keep(mask, leaf)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    r = torch.Generator().manual_seed(1)
    K0, V0 = b.K.clone(), b.V.clone()
    for turn in range(4):
        new = [20, 9, 33] if turn % 2 else [33, 20, 9]
        starts = [0, new[0], new[0] + new[1], sum(new)]
        b.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
        parents[:62] = torch.cat([torch.tensor([int(torch.randint(-1, max(i, 1), (1,), generator=r)) for i in range(n)], dtype=torch.int32) for n in new]).cuda()
        leaf.copy_(torch.tensor([n - 1 - turn for n in new], dtype=torch.int32))
        fused.copy_(_rows(b.T, 12, 10 + turn))
        b.K.copy_(K0)
        b.V.copy_(V0)
        graph.replay()
        torch.cuda.synchronize()
        seen = [x.clone() for x in got] + [b.K.clone(), b.V.clone()]
        b.K.copy_(K0)
        b.V.copy_(V0)
        want = list(step()) + [b.K, b.V]
        rows = slice(0, 62)
        for i, (x, y) in enumerate(zip(seen, want)):
            x, y = (x, y) if i >= 4 else (x[rows], y[rows])
            assert torch.equal(x.view(torch.int16) if x.dtype is torch.bfloat16 else x, y.view(torch.int16) if y.dtype is torch.bfloat16 else y), (turn, i)


def test_arguments_that_do_not_fit_are_refused():
    mp = _mp()
    b = Batch([3], [20], 2, 16)
    paged, q = b.paged(), _rows(3, 4, 1)
    good = torch.ones(3, 1, dtype=torch.int64, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")      # noqa: E731
    w = torch.ones(2, 128, dtype=torch.bfloat16, device="cuda")
    rot, x = mp.MpRotary(), _rows(3, 2, 2)
    pool = mp.MpPagePool(i32(2, 4), i32(2), i32(3), i32(8), i32(1), 16)
    for call in (
        lambda: paged.mp_paged_tree_attention(q, good.int()), lambda: paged.mp_paged_tree_attention(q, good[:2]), lambda: paged.mp_paged_tree_attention(q, good[:, 0]),
        lambda: paged.mp_paged_tree_attention(q, good.cpu()), lambda: paged.mp_paged_tree_attention(q, torch.ones(3, 17, dtype=torch.int64, device="cuda")),
        lambda: paged.mp_paged_tree_attention(q, good.expand(3, 2)), lambda: paged.mp_paged_tree_plan(i32(3, 1)), lambda: paged.mp_paged_tree_plan(i32(3).long()),
        lambda: paged.mp_paged_tree_plan(i32(3), 17), lambda: paged.mp_paged_tree_plan(i32(3), 0), lambda: paged.mp_paged_tree_plan(i32(3), 1, good[:2]),
        lambda: paged.mp_paged_tree_plan(i32(6)[::2]), lambda: paged.mp_paged_tree_keep(good, i32(2)), lambda: paged.mp_paged_tree_keep(good, i32(1).long()),
        lambda: paged.mp_paged_tree_keep(good, i32(1), i32(2)), lambda: paged.mp_paged_tree_keep(good, i32(1), b.kv_len), lambda: mp.MpHeadNorm(w.float()), lambda: mp.MpHeadNorm(w[:, :64]),
        lambda: mp.MpHeadNorm(w.cpu()), lambda: mp.MpHeadNorm(w.T), lambda: rot.mp_norm_rotary(mp.MpHeadNorm(w, eps=0.0), x, i32(3)),
        lambda: rot.mp_norm_rotary(mp.MpHeadNorm(torch.cat([w, w])), x, i32(3)), lambda: rot.mp_norm_rotary(mp.MpHeadNorm(w), x, i32(2)),
        lambda: paged.mp_paged_append_norm(x, x, k_norm=mp.MpHeadNorm(torch.cat([w, w]))), lambda: paged.mp_paged_append_norm(x, x, positions=i32(2)),
        lambda: paged.mp_paged_append_norm(x, x, q=q, q_norm=mp.MpHeadNorm(w)), lambda: mp.MpPagePool(i32(2, 4), i32(2), i32(2), i32(8), i32(1), 16),
        lambda: mp.MpPagePool(i32(2, 4), i32(3), i32(3), i32(8), i32(1), 16), lambda: mp.MpPagePool(i32(2, 4), i32(2), i32(3), i32(8, 1), i32(1), 16),
        lambda: mp.MpPagePool(i32(2, 4), i32(2), i32(3), i32(8), i32(2), 16), lambda: mp.MpPagePool(i32(2, 4), i32(2), i32(3), i32(8), i32(1), 12).mp_paged_reserve(i32(2)),
        lambda: pool.mp_paged_reserve(i32(3)), lambda: pool.mp_paged_reserve(i32(2), i32(2).long()), lambda: pool.mp_paged_reserve(i32(2), granted=i32(1)),
        lambda: pool.mp_paged_reserve(i32(2), sequence=i32(5), positions=i32(4)), lambda: pool.mp_paged_reserve(i32(2), slots=i32(4)),
        lambda: pool.mp_paged_reserve(pool.tensors[1]), lambda: pool.mp_paged_reserve(i32(2), keep=pool.tensors[1]),
    ):
        with pytest.raises(mp.MpError) as e:
            call()
        assert e.value.status == mp.MP_EINVAL
    torch.cuda.synchronize()
    assert math.isfinite(float(paged.mp_paged_tree_attention(q, good).float().sum()))
