"""GPU: the paged cache -- append, attention, gather -- against the definitions in 64 bits."""
import math

import pytest
import torch

from tests.paged_util import Batch, check, gen, turn_bound, turned

pytestmark = pytest.mark.gpu


def _mp():
    from paper_2506_13059_amd import binding as mp
    return mp


def _rows(T, H, seed, scale=1.0):
    return (scale * torch.randn(T, H, 128, generator=gen(seed), device="cuda")).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("new,lens,Hq,Hkv,page,interleaved", [
    ([1], [1], 4, 1, 16, 0),
    ([1, 1, 1], [17, 32, 700], 8, 2, 16, 0),
    ([5, 0, 33, 1], [5, 40, 40, 1], 10, 2, 8, 1),
    ([300, 200], [1000, 200], 8, 8, 64, 0),
    ([3], [3], 1, 1, 1, 1),
    ([0, 0, 2, 0], [0, 3, 2, 9], 6, 3, 32, 0),
    ([1] * 131, list(range(1, 132)), 2, 1, 16, 0),
    ([1, 2] * 2500, [40 + i % 3 for i in range(5000)], 1, 1, 16, 0),
    ([4100], [4200], 32, 8, 1024, 1),
])
def test_append(new, lens, Hq, Hkv, page, interleaved):
    mp = _mp()
    print(f"case new={new[:6]} lens={lens[:6]} Hq={Hq} Hkv={Hkv} page={page} interleaved={interleaved}", flush=True)
    b = Batch(new, lens, Hkv, page, pad_front=2, pad_back=3)
    rot = mp.MpRotary(rot_dim=64, base=1e4, layout=interleaved, amplitude=1.125)
    fused = _rows(b.T, Hq + 2 * Hkv, 5)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    q_out = torch.full((b.T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    before = b.K.clone(), b.V.clone()
    b.paged().mp_paged_append(k, v, rotary=rot, q=q, q_out=q_out)
    position = torch.cat([b.positions(i) for i in range(len(new))])
    rows = slice(b.starts[0], b.starts[-1])
    for x, got, what in ((q, q_out, "q"), (k, None, "k")):
        x = x[rows]
        want = turned(x, position, rot.freqs, interleaved, 1.125)
        if got is None:
            seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
            page_at = b.table[seq, position // page].long()
            got = b.K[page_at, :, position % page]
            assert torch.equal(b.V[page_at, :, position % page], v[rows])
            b.K[page_at, :, position % page] = before[0][page_at, :, position % page]
            b.V[page_at, :, position % page] = before[1][page_at, :, position % page]
        else:
            assert (got[:b.starts[0]] == 7).all() and (got[b.starts[-1]:] == 7).all()
            got = got[rows]
        check(got, want, turn_bound(x, want, rot.freqs, interleaved, 1.125), what)
    # nothing else has changed
    assert torch.equal(b.K.view(torch.int16), before[0].view(torch.int16)) and torch.equal(b.V.view(torch.int16), before[1].view(torch.int16))


def test_append_drops_what_has_no_place():
    mp = _mp()
    b = Batch([4, 6, 3], [2, 40, 35], 2, 16)          # two of the first sequence's tokens stand before position zero
    b.table[1, 2] = -1                                # keys 32 .. 39 of the second have no page
    b.table[2, 2] = b.n_pages                         # nor have keys 32 .. 34 of the third
    k, v, q = _rows(b.T, 2, 1), _rows(b.T, 2, 2), _rows(b.T, 4, 3)
    before = b.K.clone(), b.V.clone()
    out = b.paged().mp_paged_append(k, v, q=q)        # no rotation: as they come
    assert torch.equal(out, q)
    page, slot = b.where(0, torch.arange(2, device="cuda"))
    assert torch.equal(b.K[page, :, slot], k[2:4]) and torch.equal(b.V[page, :, slot], v[2:4])
    b.K[page, :, slot], b.V[page, :, slot] = before[0][page, :, slot], before[1][page, :, slot]
    assert torch.equal(b.K.view(torch.int16), before[0].view(torch.int16)) and torch.equal(b.V.view(torch.int16), before[1].view(torch.int16))
    # a table that ends before the tokens' positions
    b.kv_len[1] = 10000
    b.paged().mp_paged_append(k[4:10].repeat(3, 1, 1)[:b.T], v[4:10].repeat(3, 1, 1)[:b.T])
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ gather
@pytest.mark.parametrize("lens,Hkv,page,first,n,interleaved", [
    ([100], 1, 16, 0, 100, 0),
    ([1000, 17, 0, 530], 2, 64, 0, 1000, 0),
    ([300, 299], 3, 8, 33, 250, 1),
    ([5000], 8, 256, 1, 4999, 0),
    ([3, 2], 1, 1, 0, 5, 1),
    ([40], 2, 32, 100, 20, 0),
])
def test_gather(lens, Hkv, page, first, n, interleaved):
    mp = _mp()
    print(f"case lens={lens} Hkv={Hkv} page={page} first={first} n={n}", flush=True)
    b = Batch([0] * len(lens), lens, Hkv, page)
    rot = mp.MpRotary(rot_dim=96, base=1e4, layout=interleaved, amplitude=3.0)
    if lens[0] > 2 * page and page > 1:
        b.table[0, 1] = -7            # a page that is gone
    k, v, look = b.paged().mp_paged_gather(n, first=first, rotary=rot, lookup_position=500)
    position = torch.arange(first, first + n, device="cuda")
    for i, length in enumerate(lens):
        have = (position < length) & torch.cat([b.there(i), torch.zeros(first + n, dtype=torch.bool, device="cuda")])[first:first + n]
        wk, wv = (torch.zeros(Hkv, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        wk[:, have], wv[:, have] = b.keys[i][:, position[have]], b.values[i][:, position[have]]
        assert torch.equal(k[i], wk) and torch.equal(v[i], wv)
        want = turned(wk.transpose(0, 1), 500 - position, rot.freqs, interleaved)
        check(look[i].transpose(0, 1), want, turn_bound(wk.transpose(0, 1), want, rot.freqs, interleaved), "lookup")
    k2, v2 = b.paged().mp_paged_gather(n, first=first)
    assert torch.equal(k2, k) and torch.equal(v2, v)


# ------------------------------------------------------------------------------------------------ attention
def _attend(b, Hq, window=0, scale=0.0, max_new=None, q_scale=2.0, label=""):
    q = _rows(b.T, Hq + 3, 11, q_scale)[:, 2:2 + Hq]
    out = torch.full((b.T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, Hq), 7.0, dtype=torch.float32, device="cuda")
    b.paged().mp_paged_attention(q, max_new=max(b.new) if max_new is None else max_new, window=window, softmax_scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    want, wlse, ob, lb = b.attention(q, window, scale)
    rows = slice(b.starts[0], b.starts[-1])
    assert (out[:b.starts[0]] == 7).all() and (out[b.starts[-1]:] == 7).all() and (lse[:b.starts[0]] == 7).all() and (lse[b.starts[-1]:] == 7).all()
    check(lse[rows], wlse[rows], lb[rows], label + " lse")
    check(out[rows], want[rows], ob[rows], label + " out")
    return q, out, lse


TOKENS = [
    ([1], [1], 1, 1), ([1], [2], 8, 16), ([1], [16], 4, 16), ([1], [17], 4, 16), ([1], [63], 2, 64), ([1], [64], 3, 64), ([1], [65], 5, 64),
    ([1], [1000], 8, 8), ([1, 1, 1, 1], [5, 700, 64, 129], 4, 16), ([1, 0, 1, 1], [300, 50, 1, 2049], 6, 32), ([1], [20000], 4, 16),
    ([1, 1], [9001, 33], 7, 128), ([1] * 70, [1 + 7 * i for i in range(70)], 4, 16), ([2, 1, 2], [100, 200, 3000], 8, 16), ([4, 3], [900, 77], 4, 64),
    ([1, 1, 1], [0, 30, 0], 4, 16), ([1] * 300, [40 + i % 50 for i in range(300)], 2, 16), ([1], [777], 1, 1024),
]


@pytest.mark.parametrize("new,lens,G,page", TOKENS)
@pytest.mark.parametrize("Hkv,window", [(1, 0), (3, 0), (2, 37)])
def test_attention_of_single_tokens(new, lens, G, page, Hkv, window):
    print(f"case new={new[:4]} lens={lens[:4]} G={G} page={page} Hkv={Hkv} window={window}", flush=True)
    _attend(Batch(new, lens, Hkv, page, pad_front=1, pad_back=2), G * Hkv, window)


CHUNKS = [
    ([17], [17], 1, 16), ([64], [64], 4, 16), ([65], [200], 4, 64), ([300], [300], 5, 32), ([31], [1031], 8, 16), ([257], [2000], 1, 16),
    ([100, 33, 1], [100, 500, 900], 4, 16), ([1, 1, 90, 1], [64, 3000, 90, 1], 2, 16), ([513], [513], 3, 128), ([40, 0, 7], [1500, 9, 7], 7, 8),
    ([700], [5000], 2, 64), ([20], [12], 4, 16), ([50, 20], [0, 20], 6, 16), ([128], [128], 8, 1), ([1025], [1025], 1, 256), ([5] * 12, [90 + 31 * i for i in range(12)], 8, 16),
]


@pytest.mark.parametrize("new,lens,G,page", CHUNKS)
@pytest.mark.parametrize("Hkv,window", [(1, 0), (2, 0), (1, 1), (2, 100)])
def test_attention_of_chunks(new, lens, G, page, Hkv, window):
    print(f"case new={new[:4]} lens={lens[:4]} G={G} page={page} Hkv={Hkv} window={window}", flush=True)
    _attend(Batch(new, lens, Hkv, page, pad_front=3, pad_back=1), G * Hkv, window)


@pytest.mark.parametrize("columns", [0, 8192], ids=["small", "room for long sequences"])
@pytest.mark.parametrize("window", [0, 65])
@pytest.mark.parametrize("G", [1, 4, 5, 8])
def test_single_tokens_beside_a_prompt(G, window, columns):
    """Sequences of few and of many new tokens in one call, pages missing, also where nothing in the batch is as long as its page table has room for."""
    b = Batch([1, 90, 0, 1, 4, 1, 17, 1], [1, 190, 40, 513, 77, 0, 17, 130], 2, 64, seed=G, pad_front=2, pad_back=3, columns=columns)
    b.table[3, 2], b.table[4, 0], b.table[7, 1] = -1, b.n_pages + 9, -5
    _attend(b, 2 * G, window)


def test_windows_of_many_single_tokens_beside_a_prompt():
    b = Batch([1] * 40 + [60] + [1] * 29, [100 + 43 * i for i in range(70)], 12, 16, pad_back=1)
    _attend(b, 12, window=1000)


def test_many_sequences_of_several_tiles():
    n = [1 + (7 * i) % 90 for i in range(150)]
    _attend(Batch(n, [k + (31 * i) % 400 for i, k in enumerate(n)], 1, 16, pad_front=5, pad_back=9), 8)
    # the line of blocks is long enough for the places in front of items
    _attend(Batch([1000, 3, 600, 1], [9000, 4000, 600, 12000], 8, 64), 32)
    _attend(Batch([1] * 40, [3000 + 411 * i for i in range(40)], 8, 16), 16)


def _random_batch(seed):
    r = torch.Generator().manual_seed(seed)
    pick = lambda *x: x[int(torch.randint(0, len(x), (1,), generator=r))]      # noqa: E731
    size = lambda hi: int(math.exp(float(torch.rand(1, generator=r)) * math.log(hi)))      # noqa: E731
    seqs, most = pick(1, 2, 3, 9, 33), pick(1, 1, 4, 12, 200, 600)
    new = [min(most, size(most + 1)) if pick(0, 1, 1, 1) else 0 for _ in range(seqs)]
    new[0] = max(new[0], 1)
    lens = [max(0, k + size(4000) - pick(1, 1, 1, 4)) for k in new]
    return dict(new=new, lens=lens, Hkv=pick(1, 2, 3), page=pick(4, 8, 16, 32, 64, 512), G=pick(1, 2, 3, 4, 5, 6, 7, 8), window=pick(0, 0, 1, 64, 333))


@pytest.mark.parametrize("seed", range(40))
def test_random_batches(seed):
    c = _random_batch(seed)
    print("case", {**c, "new": c["new"][:6], "lens": c["lens"][:6]}, flush=True)
    b = Batch(c["new"], c["lens"], c["Hkv"], c["page"], seed=seed, pad_front=seed % 3, pad_back=seed % 2)
    if seed % 3 == 0:
        b.table[(torch.rand(b.table.shape, generator=torch.Generator().manual_seed(seed)) < 0.1).cuda()] = -1
    _attend(b, c["Hkv"] * c["G"], c["window"])


@pytest.mark.parametrize("new,lens", [([1, 1], [3000, 2000]), ([70, 1], [400, 2000]), ([260], [4000])])
def test_missing_pages_take_no_part(new, lens):
    b = Batch(new, lens, 2, 16)
    for i, n in enumerate(lens):
        e = torch.randperm(n // 16, generator=torch.Generator().manual_seed(i))[:n // 48]
        b.table[i, e.cuda()] = torch.tensor([-1, b.n_pages, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")[torch.arange(len(e), device="cuda") % 4]
    _attend(b, 8)
    _attend(b, 8, window=50)
    b.table[0] = -1                      # nothing left of the first: its rows are empty
    q, out, lse = _attend(b, 8)
    assert (out[:new[0]] == 0).all() and (lse[:new[0]] == -math.inf).all()


@pytest.mark.parametrize("new,lens", [([1], [5000]), ([6], [900]), ([100], [700])])
def test_sharp_and_large_logits(new, lens):
    b = Batch(new, lens, 2, 16, scale=4.0)
    _attend(b, 8, q_scale=8.0)           # logits of a few hundred
    _attend(b, 8, q_scale=0.0)           # all the same
    _attend(b, 8, scale=0.01)


def test_values_that_are_not_finite_stay_in_their_dimension_and_behind_their_row():
    for new, lens in (([1], [700]), ([80], [700]), ([80], [80])):
        b = Batch(new, lens, 1, 16)
        n = lens[0]
        clean = _attend(b, 4)[1]
        b.values[0][0, n - 1, 5], b.values[0][0, n - 1, 9], b.values[0][0, n - 1, 11] = math.inf, -math.inf, math.nan
        b.write()
        q = _rows(b.T, 7, 11, 2.0)[:, 2:6]
        out = b.paged().mp_paged_attention(q, max_new=new[0])
        rest = [d for d in range(128) if d not in (5, 9, 11)]
        assert torch.equal(out[..., rest], clean[..., rest])
        assert not out[-1][:, [5, 9, 11]].isfinite().any()                      # (the last token attends it)
        assert torch.equal(out[:-1][..., [5, 9, 11]], clean[:-1][..., [5, 9, 11]])  # (those before it do not)


@pytest.mark.parametrize("new,G", [([1], 4), ([4], 8), ([8], 8), ([100], 4)])
def test_infinite_values_make_their_dimension_infinite(new, G):
    b = Batch(new, [700], 1, 16)
    clean = _attend(b, G)[1]
    b.values[0][0, 10, 5], b.values[0][0, 300, 9], b.values[0][0, 300, 11] = math.inf, -math.inf, math.nan      # (older keys, which every row sees)
    b.values[0][0, 20, 13], b.values[0][0, 21, 13] = math.inf, -math.inf
    b.write()
    out = b.paged().mp_paged_attention(_rows(b.T, G + 3, 11, 2.0)[:, 2:2 + G], max_new=new[0])
    rest = [d for d in range(128) if d not in (5, 9, 11, 13)]
    assert torch.equal(out[..., rest], clean[..., rest])
    assert (out[..., 5] == math.inf).all() and (out[..., 9] == -math.inf).all() and out[..., [11, 13]].isnan().all()


def test_rows_of_the_same_values_give_them_back():
    # the weights sum to one, whatever the split
    for new, lens in (([1], [30001]), ([3], [4001]), ([200], [3001])):
        b = Batch(new, lens, 2, 64)
        b.values[0][:] = torch.randn(128, generator=gen(3), device="cuda").to(torch.bfloat16)
        b.write()
        out = b.paged().mp_paged_attention(_rows(b.T, 8, 4), max_new=new[0])
        assert ((out.double() - b.values[0][0, 0].double()).abs() <= 2.0 ** -7 * b.values[0][0, 0].double().abs()).all()


def test_one_token_at_a_time_is_the_chunk():
    # the same rows through the kernels for chunks and for single tokens: both are within their bounds of the same values
    b = Batch([40], [333], 2, 16)
    q, out, lse = _attend(b, 16)
    _, wlse, ob, lb = b.attention(q)
    for i in (0, 1, 17, 39):
        one = Batch([1], [294 + i], 2, 16)
        one.keys, one.values = [b.keys[0][:, :294 + i]], [b.values[0][:, :294 + i]]
        one.write()
        o = one.paged().mp_paged_attention(q[i:i + 1], max_new=1)
        assert ((o[0].double() - out[i].double()).abs() <= 2 * ob[i]).all()


@pytest.mark.parametrize("new", [1, 9, 150])
def test_results_repeat_and_follow_a_captured_graph(new):
    mp = _mp()
    b = Batch([new, 1], [900, 400], 2, 16)
    paged = b.paged()
    q = _rows(b.T, 8, 5)
    out, lse = torch.empty_like(q), torch.empty(b.T, 8, dtype=torch.float32, device="cuda")
    ws = [torch.full((max(1, mp.mp_paged_workspace_bytes(b.T, 8, 2, 2, new)),), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    call = lambda w: paged.mp_paged_attention(q, max_new=new, out=out, lse=lse, workspace=w)      # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(ws[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call(ws[0])
    for lens in ((900, 400), (850, 399), (new, 1), (900, 2)):
        b.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        out.fill_(0), lse.fill_(0)
        call(ws[1])
        assert torch.equal(out, got) and torch.equal(lse, got_lse)


def test_max_new_bounds_the_rows():
    b = Batch([3, 30], [50, 60], 1, 16)
    q = _rows(b.T, 4, 5)
    out = torch.full_like(q, 7.0)
    b.paged().mp_paged_attention(q, max_new=3, out=out)
    want = b.paged().mp_paged_attention(q)
    _, _, ob, _ = b.attention(q)
    assert ((out[:6].double() - want[:6].double()).abs() <= 2 * ob[:6]).all() and (out[6:] == 7).all()


def test_shared_pages():
    b = Batch([1, 1], [64, 64], 2, 16)
    b.table[1] = b.table[0]
    b.keys[1], b.values[1] = b.keys[0], b.values[0]
    q = _rows(2, 8, 5)
    q[1] = q[0]
    out = b.paged().mp_paged_attention(q, max_new=1)
    assert torch.equal(out[0], out[1])


def test_caches_of_more_than_32_bits():
    # 5.4 GB of keys and as many of values: the sequence's pages are the last ones, and the first
    mp = _mp()
    n_pages, Hkv, page, n = 41000, 8, 64, 300
    K, V = (torch.empty(n_pages, Hkv, page, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert K.numel() * 2 > 1 << 32
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, 32768, n_pages - 3]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    big = mp.MpPagedKv(K, V, table, torch.tensor([n], dtype=torch.int32, device="cuda"), starts)
    b = Batch([n], [n], Hkv, page)
    k, v = b.keys[0].transpose(0, 1).contiguous(), b.values[0].transpose(0, 1).contiguous()
    big.mp_paged_append(k, v)
    gk, gv = big.mp_paged_gather(n)
    assert torch.equal(gk[0], b.keys[0]) and torch.equal(gv[0], b.values[0])
    q = _rows(n, 16, 3, 2.0)
    assert torch.equal(big.mp_paged_attention(q), b.paged().mp_paged_attention(q))
    one = mp.MpPagedKv(K, V, table, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    out = one.mp_paged_attention(q[-1:], max_new=1)
    b1 = Batch([1], [n], Hkv, page)
    b1.keys, b1.values = b.keys, b.values
    b1.write()
    assert torch.equal(out, b1.paged().mp_paged_attention(q[-1:], max_new=1))


def test_refusals():
    mp = _mp()
    b = Batch([2], [20], 2, 16)
    p, q, k = b.paged(), _rows(2, 8, 1), _rows(2, 2, 2)
    short = torch.empty(8, dtype=torch.uint8, device="cuda")
    calls = [lambda: p.mp_paged_append(k, k[:1]), lambda: p.mp_paged_append(q, q), lambda: p.mp_paged_append(k.float(), k), lambda: p.mp_paged_append(k, k, q=q[:1]),
             lambda: p.mp_paged_append(k, k, q_out=q), lambda: p.mp_paged_append(k, k, q=q, q_out=torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")),
             lambda: p.mp_paged_attention(q[:, :7]), lambda: p.mp_paged_attention(q.float()), lambda: p.mp_paged_attention(q, lse=torch.empty(2, 8, device="cuda").double()),
             lambda: p.mp_paged_attention(q, out=q[:1]), lambda: p.mp_paged_attention(q, window=-1), lambda: p.mp_paged_attention(q, max_new=-1),
             lambda: p.mp_paged_attention(q.cpu()), lambda: p.mp_paged_attention(_rows(2, 18, 1)),
             lambda: p.mp_paged_gather(3, lookup_position=1), lambda: p.mp_paged_gather(-1), lambda: p.mp_paged_gather(3, first=-1),
             lambda: p.mp_paged_gather(3, k=b.K), lambda: p.mp_paged_gather(3, k_lookup=b.K),
             lambda: mp.MpPagedKv(b.K, b.V[:1], b.table, b.kv_len, b.q_start), lambda: mp.MpPagedKv(b.K, b.V, b.table.long(), b.kv_len, b.q_start),
             lambda: mp.MpPagedKv(b.K, b.V, b.table, b.kv_len, b.kv_len), lambda: mp.MpPagedKv(b.K, b.V, b.table[:, ::2], b.kv_len, b.q_start),
             lambda: mp.MpPagedKv(b.K[..., :64], b.V[..., :64], b.table, b.kv_len, b.q_start),
             lambda: mp.MpPagedKv(b.K[:, :, :12].contiguous(), b.V[:, :, :12].contiguous(), b.table, b.kv_len, b.q_start).mp_paged_attention(q)]
    if mp.mp_paged_workspace_bytes(2, 8, 2, 1, 2) > 8:
        calls.append(lambda: p.mp_paged_attention(q, workspace=short))
    for i, call in enumerate(calls):
        with pytest.raises(mp.MpError) as e:
            call()
        assert e.value.status == mp.MP_EINVAL, i
    assert p.mp_paged_attention(q[:0]).shape == (0, 8, 128) and p.mp_paged_gather(0)[0].shape == (1, 2, 0, 128)
