"""GPU: trees of drafted tokens over the paged cache -- ancestors and positions, attention, the accepted path's rows -- against the definitions, and a run of all of it."""
import math

import pytest
import torch

from tests.paged_util import BF16, Batch, check, gen, turned
from tests.test_gpu_norm_rotary import bound as rows_bound
from tests.test_gpu_norm_rotary import normed
from tests.tree_util import ancestors, random_parents, tree_attention, words_of

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


def _rows(T, H, seed, scale=1.0):
    return (scale * torch.randn(T, H, 128, generator=gen(seed), device="cuda")).to(torch.bfloat16)


def _mask(b, marked, words, fill=-1):
    """int64 [T, words]; rows of no sequence: `fill`."""
    rows = [[fill] * words for _ in range(b.T)]
    for s, of in enumerate(marked):
        for i, m in enumerate(of):
            rows[b.starts[s] + i] = words_of(m, words)
    return torch.tensor(rows, dtype=torch.int64, device="cuda").view(b.T, words)


# ------------------------------------------------------------------------------------------------ plan
@pytest.mark.parametrize("new,words,deep", [
    ([1], 1, 0.5), ([5, 0, 64, 3], 1, 0.5), ([64], 1, 1.0), ([65, 128, 7], 2, 0.3), ([130], 3, 0.9), ([250] * 9, 4, 0.5), ([256, 1], 4, 1.0), ([300, 512], 8, 0.2),
    ([1000], 16, 0.99), ([1024, 700], 16, 0.0), ([12] * 300, 1, 0.4), ([70, 10], 1, 0.5), ([200], 2, 0.5),
])
def test_plan(new, words, deep):
    print(f"case new={new[:5]} words={words} deep={deep}", flush=True)
    lens = [n + 11 * i for i, n in enumerate(new)]
    lens[-1] -= 2                                 # more tokens than keys: positions begin below zero
    b = Batch(new, lens, 1, 16, pad_front=2, pad_back=3)
    parents = [random_parents(n, 7 * s + 1, deep) for s, n in enumerate(new)]
    for p in parents:
        if len(p) > 4:
            p[3], p[4] = -9, 4                    # no token before it: none
    at = torch.tensor([0, 5] + sum(parents, []) + [1, 1, 1], dtype=torch.int32, device="cuda")
    mask, positions = torch.full((b.T, words), 77, dtype=torch.int64, device="cuda"), torch.full((b.T,), 77, dtype=torch.int32, device="cuda")
    b.paged().mp_paged_tree_plan(at, words, mask, positions)
    want_mask, want_pos = [[77] * words for _ in range(b.T)], [77] * b.T
    for s, p in enumerate(parents):
        for i in range(min(new[s], 64 * words)):
            path = ancestors(p, i)
            want_mask[b.starts[s] + i] = words_of(path, words)
            want_pos[b.starts[s] + i] = lens[s] - new[s] + len(path) - 1
    assert positions.tolist() == want_pos and mask.tolist() == want_mask


# ------------------------------------------------------------------------------------------------ attention
def _attend(b, Hq, marked, words, window=0, scale=0.0, max_new=None, label="", q_scale=2.0):
    q = _rows(b.T, Hq + 3, 11, q_scale)[:, 2:2 + Hq]
    out = torch.full((b.T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, Hq), 7.0, dtype=torch.float32, device="cuda")
    b.paged().mp_paged_tree_attention(q, _mask(b, marked, words), max_new=max(b.new) if max_new is None else max_new, window=window, softmax_scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    want, wlse, ob, lb = tree_attention(b, q, marked, window, scale)
    rows = slice(b.starts[0], b.starts[-1])
    assert (out[:b.starts[0]] == 7).all() and (out[b.starts[-1]:] == 7).all() and (lse[:b.starts[0]] == 7).all() and (lse[b.starts[-1]:] == 7).all()
    check(lse[rows], wlse[rows], lb[rows], label + " lse")
    check(out[rows], want[rows], ob[rows], label + " out")
    return q, out, lse


def _trees(new, seed=0, deep=0.5):
    return [[ancestors(p, i) for i in range(n)] for s, n in enumerate(new) for p in [random_parents(n, 13 * s + seed, deep)]]


TREES = [
    ([1], [1], 1, 16), ([2], [2], 8, 16), ([3], [40], 4, 16), ([12], [4096], 4, 16), ([12], [12], 4, 64), ([16], [77], 4, 1), ([7, 0, 2, 3], [300, 50, 2, 2049], 5, 32),
    ([31], [1000], 2, 8), ([64], [64], 1, 16), ([64], [65], 1, 128), ([33, 5], [2100, 5], 1, 64), ([8] * 70, [8 + 17 * i for i in range(70)], 2, 16), ([4, 4, 4], [2, 30, 4], 4, 16),
    # more than 64 query rows a head: by the kernel for chunks
    ([65], [65], 1, 16), ([24], [3000], 8, 64), ([63, 20, 63], [5000, 333, 70], 4, 64), ([250], [1300], 4, 16), ([130, 1, 7], [131, 900, 7], 5, 4), ([40, 50], [12, 20], 3, 16),
    ([1, 100, 1, 3], [2000, 700, 1, 64], 8, 16), ([700], [900], 1, 256), ([128] * 5, [128 + 63 * i for i in range(5)], 7, 8), ([17], [64 * 16], 8, 1024),
]


@pytest.mark.parametrize("new,lens,G,page", TREES)
@pytest.mark.parametrize("Hkv,window", [(1, 0), (2, 0), (1, 1), (2, 5), (1, 100)])
def test_attention_of_trees(new, lens, G, page, Hkv, window):
    print(f"case new={new[:4]} lens={lens[:4]} G={G} page={page} Hkv={Hkv} window={window}", flush=True)
    b = Batch(new, lens, Hkv, page, pad_front=1, pad_back=2)
    _attend(b, G * Hkv, _trees(new), -(-max(new) // 64), window)


@pytest.mark.parametrize("new,lens,G,page", TREES)
@pytest.mark.parametrize("window", [0, 3, 70])
def test_attention_of_any_marks(new, lens, G, page, window):
    """Masks that are no trees: tokens behind the row, none at all, some without itself, all; words that no token needs, bits behind the last token."""
    print(f"case new={new[:4]} lens={lens[:4]} G={G} page={page} window={window}", flush=True)
    g = torch.Generator().manual_seed(5)
    marked = []
    for n in new:
        of = []
        for i in range(n):
            share = [0.0, 0.1, 0.5, 1.0][int(torch.randint(0, 4, (1,), generator=g))]
            of.append([j for j in range(n) if float(torch.rand(1, generator=g)) < share] + [n, n + 1, n + 70])
        marked.append(of)
    b = Batch(new, lens, 2, page, pad_front=1, pad_back=2)
    _attend(b, G * 2, marked, min(16, -(-max(new) // 64) + 1), window)


@pytest.mark.parametrize("new,lens,G", [([6], [200], 4), ([70, 2], [200, 90], 4), ([30], [30], 1)])
def test_a_causal_mask_is_causal_attention(new, lens, G):
    for window in (0, 9):
        b = Batch(new, lens, 2, 16)
        words = -(-max(new) // 64)
        marked = [[list(range(i + 1)) for i in range(n)] for n in new]
        q, out, lse = _attend(b, 2 * G, marked, words, window)
        lse2 = torch.empty_like(lse)
        out2 = b.paged().mp_paged_attention(q, max_new=max(new), window=window, lse=lse2)
        # (a tile of a tree's rows meets the keys of all new tokens, so the keys are shared out in other parts, whose sums differ in their last bits: each is within its bound of the
        # value, and they are within two of one another)
        _, _, ob, lb = tree_attention(b, q, marked, window)
        check(out2, out.double(), 2 * ob, "out")
        check(lse2, lse.double(), 2 * lb, "lse")


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    r = torch.Generator().manual_seed(seed)
    pick = lambda *x: x[int(torch.randint(0, len(x), (1,), generator=r))]      # noqa: E731
    size = lambda hi: int(math.exp(float(torch.rand(1, generator=r)) * math.log(hi)))      # noqa: E731
    seqs, most = pick(1, 2, 9, 33), pick(2, 6, 20, 130)
    new = [min(most, size(most + 1)) if pick(0, 1, 1, 1) else 0 for _ in range(seqs)]
    new[0] = max(new[0], 1)
    lens = [max(0, k + size(4000) - pick(1, 1, 1, 4)) for k in new]
    Hkv, page, G, window = pick(1, 2, 3), pick(4, 8, 16, 32, 64, 512), pick(1, 2, 3, 4, 5, 6, 7, 8), pick(0, 0, 1, 8, 333)
    print(f"case new={new[:6]} lens={lens[:6]} Hkv={Hkv} page={page} G={G} window={window}", flush=True)
    b = Batch(new, lens, Hkv, page, seed=seed, pad_front=seed % 3, pad_back=seed % 2, columns=pick(0, 0, 3000))
    if seed % 3 == 0:
        b.table[(torch.rand(b.table.shape, generator=torch.Generator().manual_seed(seed)) < 0.1).cuda()] = -1
    _attend(b, Hkv * G, _trees(new, seed, pick(0.0, 0.5, 0.95)), -(-max(new) // 64), window, max_new=pick(max(new), b.T))


@pytest.mark.parametrize("new,lens,G", [([12], [300], 4), ([12], [300], 8), ([70], [300], 4), ([6], [6], 2)])
def test_what_a_token_does_not_mark_may_hold_anything(new, lens, G):
    b = Batch(new, lens, 2, 16)
    marked = [[[j for j in m if j % 3 != 1] for m in of] for of in _trees(new)]
    q, out, lse = _attend(b, 2 * G, marked, 2)
    n, older = new[0], lens[0] - new[0]
    for x, y in ((float("nan"), float("inf")), (float("inf"), float("nan"))):
        for j in range(1, n, 3):
            page, slot = b.where(0, torch.tensor(older + j, device="cuda"))
            b.K[page, :, slot], b.V[page, :, slot] = x, y
        lse2 = torch.empty_like(lse)
        out2 = b.paged().mp_paged_tree_attention(q, _mask(b, marked, 2), max_new=n, lse=lse2)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("new,G", [(12, 4), (12, 8), (70, 2)])
def test_infinite_values_reach_the_tokens_that_mark_them(new, G):
    b = Batch([new], [new + 90], 1, 16)
    marked = _trees([new])
    j = 3
    b.values[0][:, 90 + j, 17] = math.inf
    b.write()
    q = _rows(new, G, 1)
    out = b.paged().mp_paged_tree_attention(q, _mask(b, marked, 2), max_new=new)
    sees = torch.tensor([j in m for m in marked[0]], device="cuda")
    assert (out[sees][:, :, 17] == math.inf).all() and out[~sees].isfinite().all()
    out[:, :, 17] = 0
    assert out.isfinite().all()


@pytest.mark.parametrize("new,G", [(1, 4), (4, 4), (8, 2), (5, 4), (8, 4), (9, 4), (16, 4), (17, 4), (32, 4), (33, 4), (63, 4), (100, 8)])
@pytest.mark.parametrize("seqs", [1, 3])
def test_nothing_is_written_past_the_workspace(new, G, seqs):
    mp = _mp()
    b = Batch([new] * seqs, [2000 + new] * seqs, 2, 16)
    n = mp.mp_paged_workspace_bytes(b.T, 2 * G, 2, seqs, new)
    whole = torch.full((n + (64 << 20),), 85, dtype=torch.uint8, device="cuda")       # (room behind it for the largest kernel's parts)
    q = _rows(b.T, 2 * G, 3)
    out = b.paged().mp_paged_tree_attention(q, _mask(b, _trees(b.new), -(-new // 64)), max_new=new, workspace=whole[:n])
    assert (whole[n:] == 85).all()
    want, _, ob, _ = tree_attention(b, q, _trees(b.new))
    check(out, want, ob, "out")


def test_workspace_that_is_shared_and_repeated_calls():
    mp = _mp()
    b = Batch([24, 9, 24], [3000, 100, 777], 4, 16)
    marked = _trees(b.new)
    q = _rows(b.T, 32, 3)
    ws = torch.full((mp.mp_paged_workspace_bytes(b.T, 32, 4, 3, 24),), 255, dtype=torch.uint8, device="cuda")
    want = b.paged().mp_paged_tree_attention(q, _mask(b, marked, 1), max_new=24)
    for _ in range(3):
        assert torch.equal(b.paged().mp_paged_tree_attention(q, _mask(b, marked, 1), max_new=24, workspace=ws), want)


# ------------------------------------------------------------------------------------------------ the accepted path
@pytest.mark.parametrize("new,lens,Hkv,page,words", [
    ([1], [1], 1, 16, 1), ([12], [4096], 8, 16, 1), ([5, 0, 33, 64], [5, 40, 40, 900], 3, 8, 1), ([250, 31], [1000, 31], 2, 64, 4), ([1000], [2000], 1, 1, 16),
    ([20] * 65, [20 + 7 * i for i in range(65)], 5, 32, 1), ([9, 9], [4, 9], 2, 16, 1),
])
@pytest.mark.parametrize("deep", [0.3, 0.95])
def test_keep(new, lens, Hkv, page, words, deep):
    print(f"case new={new[:4]} lens={lens[:4]} Hkv={Hkv} page={page} deep={deep}", flush=True)
    b = Batch(new, lens, Hkv, page, pad_front=2, pad_back=1)
    if lens[0] > 2 * page and page > 1:
        b.table[0, (lens[0] - 2) // page] = -1              # the last tokens' page is gone
    marked = _trees(new, 3, deep)
    g = torch.Generator().manual_seed(3)
    leaf = [int(torch.randint(-1, n + 1, (1,), generator=g)) if i % 3 == 2 else n - 1 for i, n in enumerate(new)]
    mask = _mask(b, marked, words)
    wantK, wantV, keep = b.K.clone(), b.V.clone(), []
    for s, n in enumerate(new):
        older = lens[s] - n
        path = [j for j in marked[s][leaf[s]] if j < 64 * words] if 0 <= leaf[s] < n else []
        keep.append(max(0, older + len(path)))
        there = b.there(s).tolist()
        for i, j in enumerate(path):
            if i != j and older + i >= 0 and there[older + i] and there[older + j]:
                p, q = b.where(s, torch.tensor(older + i, device="cuda")), b.where(s, torch.tensor(older + j, device="cuda"))
                wantK[p[0], :, p[1]], wantV[p[0], :, p[1]] = b.K[q[0], :, q[1]], b.V[q[0], :, q[1]]
    got = b.paged().mp_paged_tree_keep(mask, torch.tensor(leaf, dtype=torch.int32, device="cuda"))
    assert got.tolist() == keep
    assert torch.equal(b.K.view(torch.int16), wantK.view(torch.int16)) and torch.equal(b.V.view(torch.int16), wantV.view(torch.int16))
    assert b.kv_len.tolist() == lens


# ------------------------------------------------------------------------------------------------ a run of it all
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_a_speculating_server(captured):
    """Prompts, then steps of drafted trees: pages reserved, ancestors planned, rows normed, turned and appended, attended, the accepted path kept, pages of the rest given back.
    captured: a step is recorded once and replayed on what the program writes into its inputs."""
    mp = _mp()
    seqs, Hq, Hkv, page, columns, most, eps = 3, 8, 2, 16, 20, 11, 1e-6
    G, n_pages = Hq // Hkv, 40
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")      # noqa: E731
    table = torch.full((seqs, columns), -1, dtype=torch.int32, device="cuda")
    kv_len, q_start, n_free = i32(seqs), i32(seqs + 1), torch.full((1,), n_pages, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).int().cuda()
    K, V = (torch.full((n_pages, Hkv, page, 128), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pool, cache = mp.MpPagePool(table, kv_len, q_start, free, n_free, page), mp.MpPagedKv(K, V, table, kv_len, q_start)
    rot = mp.MpRotary(base=1e4)
    wq, wk = ((1 + 0.2 * torch.randn(128, generator=gen(s), device="cuda")).to(torch.bfloat16) for s in (1, 2))
    q_norm, k_norm = mp.MpHeadNorm(wq, eps=eps), mp.MpHeadNorm(wk, eps=eps)
    T = seqs * most
    n_new, keep, leaf, granted, parents = i32(seqs), i32(seqs), i32(seqs), i32(seqs), i32(T)
    mask, positions = torch.zeros(T, 1, dtype=torch.int64, device="cuda"), i32(T)
    fused, out, turned_q = (torch.zeros(T, h, 128, dtype=torch.bfloat16, device="cuda") for h in (Hq + 2 * Hkv, Hq, Hq))
    ws = torch.empty(mp.mp_paged_workspace_bytes(T, Hq, Hkv, seqs, most), dtype=torch.uint8, device="cuda")

    def draft():
        pool.mp_paged_reserve(n_new, keep, granted)
        cache.mp_paged_tree_plan(parents, 1, mask, positions)
        cache.mp_paged_append_norm(fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:], rotary=rot, q=fused[:, :Hq], q_out=turned_q, q_norm=q_norm, k_norm=k_norm, positions=positions)
        cache.mp_paged_tree_attention(turned_q, mask, max_new=most, out=out, workspace=ws)

    def accept():
        cache.mp_paged_tree_keep(mask, leaf, keep)

    # prompts, of rows that the program appends in order
    have = [37, 5, 64]
    n_new.copy_(torch.tensor(have, dtype=torch.int32))
    pool.mp_paged_reserve(n_new, keep)
    rows = _rows(sum(have), Hq + 2 * Hkv, 9)
    cache.mp_paged_append_norm(rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], rotary=rot, k_norm=k_norm)
    model = [list(rows[sum(have[:s]):sum(have[:s + 1])]) for s in range(seqs)]
    keep.copy_(kv_len)
    graphs = None
    if captured:
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for g, f in zip(graphs, (draft, accept)):
            with torch.cuda.graph(g):
                f()
    r = torch.Generator().manual_seed(4)
    for step in range(6):
        new = [int(torch.randint(1, most + 1, (1,), generator=r)) for _ in range(seqs)]
        if step == 4:
            model[1], new[1] = [], 8                 # a sequence ends, another one takes its place
            keep[1] = 0
        trees = [random_parents(n, 100 * step + s) for s, n in enumerate(new)]
        n_new.copy_(torch.tensor(new, dtype=torch.int32))
        parents[:sum(new)] = torch.tensor(sum(trees, []), dtype=torch.int32, device="cuda")
        fused.copy_(_rows(T, Hq + 2 * Hkv, 50 + step))
        graphs[0].replay() if captured else draft()
        torch.cuda.synchronize()
        assert granted.tolist() == new
        at = 0
        leaves = []
        for s, n in enumerate(new):
            for i in range(n):
                path = ancestors(trees[s], i)
                line = torch.stack(model[s] + [fused[at + j] for j in path])                      # all that the token attends, in order
                pos, older = torch.arange(line.shape[0], device="cuda"), len(model[s])
                # rows in the cache and queries as they were made, each near the formula's, then attention of just these
                place = torch.tensor(list(range(older)) + [older + j for j in path], device="cuda")
                page_at, slot = table[s].long()[place // page], place % page
                k, v, q = K[page_at, :, slot], V[page_at, :, slot], turned_q[at + i:at + i + 1]
                for got, x, w, p in ((k, line[:, Hq:Hq + Hkv], wk, pos), (q, line[-1:, :Hq], wq, pos[-1:])):
                    xn = normed(x, w, 0.0, eps)
                    want = turned(xn, p, rot.freqs, 0)
                    check(got, want, rows_bound(xn, want, rot.freqs, 0), f"step {step} sequence {s} token {i}")
                assert torch.equal(v, line[:, Hq + Hkv:])
                for h in range(Hq):
                    x, kh, vh = q[0, h].double(), k[:, h // G].double(), v[:, h // G].double()
                    p = torch.softmax(kh @ x / math.sqrt(128), 0)
                    d = 130 * 2.0 ** -24 * float(x.norm() * kh.norm(dim=1).max()) / math.sqrt(128)
                    bound = BF16 * (p @ vh).abs() + (BF16 + 2 * d + (len(pos) + 64) * 2.0 ** -24) * (p @ vh.abs())      # (as in tree_attention)
                    assert ((out[at + i, h].double() - p @ vh).abs() <= bound).all(), (step, s, i, h)
            leaves.append(int(torch.randint(0, n, (1,), generator=r)))
            model[s] = model[s] + [fused[at + j].clone() for j in ancestors(trees[s], leaves[-1])]
            at += n
        leaf.copy_(torch.tensor(leaves, dtype=torch.int32))
        graphs[1].replay() if captured else accept()
        assert keep.tolist() == [len(m) for m in model]
    # what is left in the cache are the accepted rows in order
    pool.mp_paged_reserve(i32(seqs), keep)
    assert kv_len.tolist() == [len(m) for m in model] and int(n_free) == n_pages - sum(-(-len(m) // page) for m in model)
    n = max(len(m) for m in model)
    k, v = cache.mp_paged_gather(n)
    for s, m in enumerate(model):
        line = torch.stack(m)
        want = turned(normed(line[:, Hq:Hq + Hkv], wk, 0.0, eps), torch.arange(len(m), device="cuda"), rot.freqs, 0)
        assert torch.equal(v[s, :, :len(m)], line[:, Hq + Hkv:].transpose(0, 1))
        check(k[s, :, :len(m)].transpose(0, 1), want, rows_bound(normed(line[:, Hq:Hq + Hkv], wk, 0.0, eps), want, rot.freqs, 0), "keys")
