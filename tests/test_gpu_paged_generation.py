"""GPU: rotary positions, the paged cache and the clustered index together, as a server runs them: prompts are read into pages piece by piece,
their rows become an index, and tokens are decoded over it."""
import math

import pytest
import torch

from tests.paged_util import check, gen, turned

pytestmark = pytest.mark.gpu

SCALE = 1.0 / math.sqrt(128)


def _attention(q, k, v, first):
    """q [tokens, Hq, 128] at positions first .. over k, v [Hkv, keys, 128], all fp64 -> out, sum of weights times |v|"""
    G = q.shape[1] // k.shape[0]
    out, size = torch.empty_like(q), torch.empty_like(q)
    seen = torch.arange(k.shape[1], device=q.device)[None] <= first + torch.arange(q.shape[0], device=q.device)[:, None]
    for h in range(q.shape[1]):
        w = torch.softmax((q[:, h] @ k[h // G].t().contiguous() * SCALE).masked_fill(~seen, -math.inf), dim=1)
        out[:, h], size[:, h] = w @ v[h // G], w @ v[h // G].abs()
    return out, size


@pytest.mark.parametrize("interleaved,lookup", [(0, True), (1, False)])
def test_prompts_index_and_decode(interleaved, lookup):
    from paper_2506_13059_amd import binding as mp
    Hq, Hkv, page, n, B = 8, 2, 16, 700, 2
    AT = 300                                                    # where lookup keys and queries stand
    rot = mp.MpRotary(rot_dim=64, base=1e4, layout=interleaved)
    n_pages = 2 * (-(-(n + 40) // page)) + 1
    K, V = (torch.full((n_pages, Hkv, page, 128), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1))[:2 * (n_pages // 2)].to(torch.int32).view(B, -1).cuda().contiguous()
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    g = gen(7)
    total = n + 24
    fused = torch.randn(B, total, Hq + 2 * Hkv, 128, generator=g, device="cuda").to(torch.bfloat16)
    position = torch.arange(total, device="cuda")
    plain_k = [turned(fused[b, :, Hq:Hq + Hkv], position, rot.freqs, interleaved).to(torch.bfloat16).double().transpose(0, 1).contiguous() for b in range(B)]
    plain_q = [turned(fused[b, :, :Hq], position, rot.freqs, interleaved).to(torch.bfloat16).double() for b in range(B)]
    values = [fused[b, :, Hq + Hkv:].double().transpose(0, 1).contiguous() for b in range(B)]
    # the prompts, in pieces of different lengths: (of the first, of the second)
    done = [0, 0]
    for piece in ((300, 1), (1, 511), (0, 100), (399, 88)):
        rows = torch.cat([fused[b, done[b]:done[b] + piece[b]] for b in range(B)])
        starts = torch.tensor([0, piece[0], piece[0] + piece[1]], dtype=torch.int32, device="cuda")
        first, done = list(done), [done[b] + piece[b] for b in range(B)]
        kv_len.copy_(torch.tensor(done, dtype=torch.int32))
        batch = mp.MpPagedKv(K, V, table, kv_len, starts)
        q = batch.mp_paged_append(rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rotary=rot, q=rows[:, :Hq])
        out = batch.mp_paged_attention(q, max_new=max(piece))
        for b in range(B):
            if piece[b]:
                part = slice(0, piece[0]) if b == 0 else slice(piece[0], sum(piece))
                want, size = _attention(plain_q[b][first[b]:done[b]], plain_k[b][:, :done[b]], values[b][:, :done[b]], first[b])
                # one rounding of the result, one of the weights, and as much again for rotated elements that fp32 rounds to bf16 the other way: one in some
                # thousand is 2^-8 of itself off then, which moves a logit by |q_d k_d| 2^-8 / sqrt(128), less than 2^-8 for any of a row's few
                check(out[part], want, 2.0 ** -8 * want.abs() + 2.0 ** -7 * size, f"piece {piece} of sequence {b}")
    assert done == [n, n]
    # what the pages hold becomes an index
    got = batch.mp_paged_gather(n, rotary=rot, lookup_position=AT) if lookup else batch.mp_paged_gather(n)
    k, v = got[0], got[1]
    for b in range(B):
        assert ((k[b].double() - plain_k[b][:, :n]).abs() <= 2.0 ** -7 * plain_k[b][:, :n].abs() + 1e-5).all()
        assert torch.equal(v[b].double(), values[b][:, :n])
    ctx = mp.MpContext(B, Hq, Hkv, max_tokens=n + 64, levels=1, max_fine=64, max_tail=64, lookup_keys=lookup)
    ctx.mp_cluster_kv(k, v, 40, iters=3, k_lookup=got[2] if lookup else None)
    ctx.mp_local_buffer_init(16)
    # tokens: over the index, with a budget for all of its keys, and over the pages
    for i in range(20):
        rows = fused[:, n + i]
        at = torch.full((B,), n + i, dtype=torch.int32, device="cuda")
        q = rot.mp_rotary(rows[:, :Hq], at, lookup_position=AT if lookup else None)
        kn = rot.mp_rotary(rows[:, Hq:Hq + Hkv], at, lookup_position=AT if lookup else None)
        (q, q_look), (kn, k_look) = (q, kn) if lookup else ((q, None), (kn, None))
        vn = rows[:, Hq + Hkv:].contiguous()
        out = ctx.mp_decode_step(q, kn.view(B, Hkv, 1, 128), vn.view(B, Hkv, 1, 128), key_budget=n + 64, q_lookup=q_look,
                                 k_new_lookup=None if k_look is None else k_look.view(B, Hkv, 1, 128))
        kv_len.fill_(n + i + 1)
        step = mp.MpPagedKv(K, V, table, kv_len, torch.arange(B + 1, dtype=torch.int32, device="cuda"))
        q_paged = step.mp_paged_append(rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rotary=rot, q=rows[:, :Hq])
        assert torch.equal(q_paged, q)
        paged = step.mp_paged_attention(q, max_new=1)
        for b in range(B):
            want, size = _attention(plain_q[b][n + i:n + i + 1], plain_k[b][:, :n + i + 1], values[b][:, :n + i + 1], n + i)
            bound = (2.0 ** -8 * want.abs() + 2.0 ** -7 * size)[0]
            check(paged[b], want[0], bound, f"token {i} of sequence {b}, pages")
            check(out[b], want[0], bound, f"token {i} of sequence {b}, index")
    ctx.close()


def test_a_captured_step_follows_its_sequences():
    """One graph of append and attention, replayed while lengths grow and pages are handed out, against eager calls on another cache."""
    from paper_2506_13059_amd import binding as mp
    Hq, Hkv, page, B = 16, 4, 16, 3
    rot = mp.MpRotary()
    table = torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
    caches = [[torch.zeros(24, Hkv, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    rows = torch.zeros(B, Hq + 2 * Hkv, 128, dtype=torch.bfloat16, device="cuda")
    batch = [mp.MpPagedKv(*c, table, kv_len, starts) for c in caches]
    q, out = (torch.empty(B, Hq, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = [torch.empty(mp.mp_paged_workspace_bytes(B, Hq, Hkv, B, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step():
        batch[0].mp_paged_append(rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rotary=rot, q=rows[:, :Hq], q_out=q)
        batch[0].mp_paged_attention(q, max_new=1, out=out, workspace=ws[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()                                              # (no sequence has a page yet: nothing is stored)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
    handed = iter(torch.randperm(24, generator=torch.Generator().manual_seed(2)).tolist())
    g = gen(5)
    for i in range(37):
        for b in range(B):
            if (i + 5 * b) % page == 0 or i == 0:
                table[b, (i + 5 * b) // page] = next(handed)
        kv_len.copy_(torch.tensor([i + 1 + 5 * b for b in range(B)], dtype=torch.int32))
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, q2 = out.clone(), batch[1].mp_paged_append(rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rotary=rot, q=rows[:, :Hq])
        want = batch[1].mp_paged_attention(q2, max_new=1, workspace=ws[1])
        assert torch.equal(q, q2) and torch.equal(got, want), i
        assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


def test_two_streams_at_once():
    from paper_2506_13059_amd import binding as mp
    from tests.paged_util import Batch
    work = []
    for i, (new, lens) in enumerate((([200, 1, 40], [3000, 900, 2000]), ([1, 1, 1], [9000, 40, 700]))):
        b = Batch(new, lens, 2, 16, seed=i)
        q = torch.randn(b.T, 16, 128, generator=gen(i), device="cuda").to(torch.bfloat16)
        work.append((b, b.paged(), q, b.paged().mp_paged_attention(q, max_new=max(new)), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        outs = []
        for b, paged, q, _, s in work:
            with torch.cuda.stream(s):
                outs.append([paged.mp_paged_attention(q, max_new=max(b.new)) for _ in range(3)])
        torch.cuda.synchronize()
        for (_, _, _, want, _), got in zip(work, outs):
            assert all(torch.equal(x, want) for x in got)
