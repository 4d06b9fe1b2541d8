"""Performance cases of the operators around speculative decoding with a paged cache.

Norms of each head's queries and keys with the rotation in the same pass (`mp_norm_rotary`, `mp_paged_append_norm`), page tables and maps
of a step's rows worked out on the GPU (`mp_paged_reserve`), and trees of drafted tokens: their ancestors and positions
(`mp_paged_tree_plan`), attention over the cache (`mp_paged_tree_attention`) and the rows of the accepted path moved together
(`mp_paged_tree_keep`).

Where `own` is false, `run` computes the same in elementary torch operations in 32 bits (angles in 64), rounded once at the end.

Keys have four channels far from zero in every head, the same way for all tokens, as key caches have them; queries of the attention
are drawn so that logits have a standard deviation of about two; values are N(0, 1).  Pages are handed out in random order.  A drafted
token's parent is one of those before it, so that trees of 60 tokens are some ten deep.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
LOOKUP_AT = 4096             # the position that lookup queries are turned to
MOST_PAIRS = 2.2e9           # (query, key, head) triples of the plain form: no drawn case has more than the largest listed one
MOST_ROWS = 16 * 8 * 66000   # key rows (times two: and value rows) of a cache
MOST_ENTRIES = 1 << 20       # of a page table


# ---------------------------------------------------------------------------------------- cases
def _case(name, kind, B, Hq, Hkv, new, context, **more):
    base = dict(name=name, kind=kind, B=B, Hq=Hq, Hkv=Hkv, new=new, context=context, ragged=False, page=16, window=0, mixed=False,
                rot=128, interleaved=False, base=1e6, factor=1.0, per_head=False, offset=0.0, eps=1e-6, fresh=0, tight=False)
    base.update(more)
    return base


def listed():
    return [
        # a decode step of sixteen sequences: queries normalised, at their own positions and at the one that centroids are scored at
        _case("norm_tokens_b16", "turn", 16, 32, 8, 1, 131072, ragged=True),
        # one token each of sixteen sequences joins the cache, queries and keys normalised: every step of a server
        _case("append_tokens_b16", "append", 16, 32, 8, 1, 32768, ragged=True),
        # five prompts' tokens of odd numbers go to pages of 64; weights of each head, kept as what they differ from one by; adjacent pairs
        _case("append_prompts_b5_g5", "append", 5, 40, 8, 4099, 20000, ragged=True, page=64, per_head=True, offset=1.0, interleaved=True, rot=64, base=1e4),
        # a step of 64 sequences: eight drafted tokens each after some of the last ones were dropped
        _case("reserve_drafts_b64", "reserve", 64, 1, 1, 8, 32768, ragged=True),
        # a step of 512 sequences, of which every eighth has ended and makes room for a new prompt
        _case("reserve_prompts_b512", "reserve", 512, 1, 1, 1021, 16384, ragged=True, fresh=8, tight=True),
        # trees of 32 drafted tokens for eight sequences
        _case("plan_32_b8", "plan", 8, 1, 1, 32, 32768, ragged=True),
        # trees of up to 250 for many
        _case("plan_250_b128", "plan", 128, 1, 1, 250, 32768, ragged=True),
        # a small tree over 4096 keys: a single user
        _case("tree_12_4k_b1", "attend", 1, 32, 8, 12, 4096),
        # eight sequences of up to 30K, groups of eight query heads, the last 4096 keys of each path
        _case("tree_24_30k_b8_g8_window", "attend", 8, 64, 8, 24, 30011, ragged=True, window=4096, page=64),
        # sixteen sequences of up to 64K with large trees: the largest call
        _case("tree_63_64k_b16", "attend", 16, 32, 8, 63, 65536, ragged=True, page=64),
        # the accepted path's rows, one layer, a single user's tree
        _case("keep_32_b1", "keep", 1, 32, 8, 32, 4096),
        # ... and of a large batch
        _case("keep_60_b192", "keep", 192, 32, 8, 60, 2048, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["turn", "append", "append", "reserve", "reserve", "plan", "attend", "attend", "attend", "keep"])
        Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
        c = _case("", kind, _log_int(rng, 1, 33), Hkv * G, Hkv, 1, _log_int(rng, 17, 131072), ragged=rng.random() < 0.7, page=rng.choice([16, 32, 64, 128, 256]))
        del c["name"]
        if kind in ("turn", "append"):
            c.update(rot=rng.choice([32, 64, 96, 128]), interleaved=rng.random() < 0.4, base=rng.choice([1e4, 5e5, 1e6]), factor=rng.choice([1.0, 4.0, 8.0]),
                     per_head=rng.random() < 0.4, offset=rng.choice([0.0, 0.0, 1.0]), eps=rng.choice([1e-6, 1e-5]), new=_log_int(rng, 1, 8192))
        elif kind == "reserve":
            c.update(B=_log_int(rng, 1, 1024), Hq=1, Hkv=1, new=_log_int(rng, 1, 2048), fresh=rng.choice([0, 0, 3, 8]), tight=rng.random() < 0.3)
        elif kind == "plan":
            c.update(B=_log_int(rng, 1, 256), Hq=1, Hkv=1, new=_log_int(rng, 2, 250))
        else:
            c.update(new=_log_int(rng, 2, 128), window=rng.choice([0, 0, 0, 1023, 4096]) if kind == "attend" else 0, mixed=kind == "attend" and rng.random() < 0.3)
        c["new"] = min(c["new"], c["context"])
        rows = c["B"] * c["Hkv"] * c["context"]
        tokens = c["B"] * c["new"] * (c["Hq"] + 2 * c["Hkv"])
        entries = c["B"] * -(-(c["context"] + c["new"]) // c["page"])
        if kind == "reserve" or kind == "plan":
            if entries <= MOST_ENTRIES and c["B"] * c["new"] <= 1 << 18 and c["B"] * c["new"] ** 2 <= 128 * 250 ** 2 * (20 if kind == "reserve" else 1):
                return c
        elif rows <= MOST_ROWS and (kind != "attend" or c["B"] * c["Hq"] * c["new"] * c["context"] <= MOST_PAIRS) and tokens <= 5 * 4099 * 56:
            return c


# ---------------------------------------------------------------------------------------- sizes of a case
def _lengths(c):
    """(new tokens, keys with them) of every sequence."""
    rng = random.Random(c["B"] * 1000003 + c["context"] * 31 + c["new"])
    new, keys = [], []
    for b in range(c["B"]):
        full = b == 0 or not c["ragged"]
        n = c["new"] if full else 1 if c["mixed"] else rng.randint(max(1, c["new"] // 2), c["new"])
        k = c["context"] if full else int(c["context"] * math.exp(rng.uniform(math.log(0.125), 0.0)))
        new.append(n)
        keys.append(max(n, k))
    return new, keys


def _requests(c):
    """Of every sequence: keys that it has, keys that stay, tokens to come."""
    new, keys = _lengths(c)
    rng = random.Random(c["B"] * 7 + c["context"] + c["new"] * 101)
    have, stay, come = [], [], []
    for b, (n, k) in enumerate(zip(new, keys)):
        ends = c["fresh"] and b % c["fresh"] == 0
        have.append(k)
        stay.append(0 if ends else k - rng.randint(0, min(n, 8) - 1) if c["new"] > 1 else k)
        come.append(n if not c["fresh"] or ends else 1)
    return have, stay, come


def _words(c):
    return -(-c["new"] // 64)


def work(c):
    new, keys = _lengths(c)
    T, Hq, Hkv, row = sum(new), c["Hq"], c["Hkv"], D * 2
    if c["kind"] == "turn":
        return {"bytes": T * Hq * row * 3 + 4 * T, "flops": T * Hq * (c["rot"] * 6 + 4 * D)}
    if c["kind"] == "append":
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * row, "flops": T * (Hq + Hkv) * (c["rot"] * 3 + 4 * D)}
    if c["kind"] == "reserve":
        have, stay, come = _requests(c)
        pages = sum(-(-(s + n) // c["page"]) - -(-s // c["page"]) for s, n in zip(stay, come))
        return {"bytes": c["B"] * 4 * 6 + 4 * 4 * pages + sum(come) * (4 + 4 + 8), "flops": 0}
    if c["kind"] == "plan":
        return {"bytes": T * (4 + 4 + 8 * _words(c)) + 8 * c["B"], "flops": 0}
    if c["kind"] == "attend":
        pairs = rows = 0
        for n, k in zip(new, keys):
            older = min(k - n, c["window"]) if c["window"] else k - n
            pairs += n * (older + 1)
            rows += older + n
        return {"bytes": rows * Hkv * 2 * row + T * (Hq * (2 * row + 4) + 8 * _words(c)), "flops": 4 * D * Hq * pairs}
    # (how deep the accepted path is depends on the tree: about 2 ln n tokens, of which some lie where they are to be)
    return {"bytes": sum(2 * math.log(n + 1) for n in new) * Hkv * 4 * row, "flops": 0}


# ---------------------------------------------------------------------------------------- inputs
def _frequencies(c):
    """Radians a position of every pair.  factor > 1: turns of a pair over the original length say how far it is slowed down."""
    d = c["rot"]
    f = c["base"] ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    if c["factor"] > 1.0:
        keep = np.clip((8192 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * keep + f / c["factor"] * (1.0 - keep)
    return f


def _amplitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["factor"] > 1.0 else 1.0


def _keys(shape, heads_at, g):
    """Keys with four large channels a head."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    far = torch.zeros(shape[heads_at], D, device="cuda")
    for h in range(shape[heads_at]):
        far[h, torch.randperm(D, generator=g, device="cuda")[:4]] = 8.0
    at = [1] * len(shape)
    at[heads_at], at[-1] = shape[heads_at], D
    return x.add_(far.view(at).to(torch.bfloat16))


def _parents(c, new, seed):
    """Of every new token, the one before it that it follows (the first of a sequence: none), counted within its sequence."""
    r = np.random.RandomState((int(seed) * 31 + 5) % (2 ** 31))
    got = []
    for n in new:
        i = np.arange(n)
        p = np.floor(i * np.sqrt(r.rand(n))).astype(np.int32)
        p[0] = -1
        got.append(p)
    return got


def _page_table(c, keys, columns, seed, spare):
    """(table, pages in no use, number of pages): pages in random order, -1 for none."""
    need = [-(-k // c["page"]) for k in keys]
    n_pages = sum(need) + spare
    table = np.full((len(keys), columns), -1, dtype=np.int32)
    order = np.random.RandomState(int(seed) % (2 ** 31)).permutation(n_pages).astype(np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table).cuda(), order[at:], n_pages


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)
    new, keys = _lengths(c)
    B, Hq, Hkv, page, T = c["B"], c["Hq"], c["Hkv"], c["page"], sum(new)
    st = dict(case=c, new=new, keys=keys, T=T)
    if own:
        from paper_2506_13059_amd import binding as mp
        st["mp"] = mp
    if c["kind"] == "reserve":
        return _prepare_reserve(c, seed, st)
    starts = np.concatenate([[0], np.cumsum(new)])
    st["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    st["kv_len"] = torch.tensor(keys, dtype=torch.int32, device="cuda")
    if c["kind"] in ("turn", "append"):
        pos = np.concatenate([np.arange(k - n, k) for n, k in zip(new, keys)])
        st["positions"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
        st["freqs"], st["amplitude"] = torch.from_numpy(_frequencies(c)).cuda(), _amplitude(c)
        # the rows of a fused projection: queries, keys, values of a token behind one another
        st["qkv"] = _keys((T, Hq + 2 * Hkv, D), 1, g)
        st["q"], st["k"], st["v"] = st["qkv"][:, :Hq], st["qkv"][:, Hq:Hq + Hkv], st["qkv"][:, Hq + Hkv:]
        for name, heads in (("q_weight", Hq), ("k_weight", Hkv)):
            w = 1.0 - c["offset"] + 0.3 * torch.randn(heads if c["per_head"] else 1, D, generator=g, device="cuda")
            st[name] = w.to(torch.bfloat16)
    if c["kind"] not in ("turn", "plan"):
        st["page_table"], _, n_pages = _page_table(c, keys, max(-(-k // page) for k in keys), seed, 3)
        st["k_pages"] = _keys((n_pages, Hkv, page, D), 1, g)
        st["v_pages"] = torch.randn(n_pages, Hkv, page, D, generator=g, device="cuda", dtype=torch.bfloat16)
    elif c["kind"] == "plan":
        # (what the plan is made for: it looks at none of the rows)
        st["page_table"], _, n_pages = _page_table(c, keys, max(-(-k // page) for k in keys), seed, 3)
        st["k_pages"] = st["v_pages"] = torch.zeros(n_pages, 1, page, D, device="cuda", dtype=torch.bfloat16)
    if c["kind"] in ("plan", "attend", "keep"):
        st["parents"] = _parents(c, new, seed)
        st["parents_at"] = torch.from_numpy(np.concatenate(st["parents"])).cuda()
        if c["kind"] != "plan":
            st["mask"] = _plain_plan(st)["mask"]
    if c["kind"] == "attend":
        st["q"] = (2.0 * torch.randn(T, Hq, D, generator=g, device="cuda")).to(torch.bfloat16)
    if c["kind"] == "keep":
        # the last accepted token of each sequence: one of the tree's second half
        r = np.random.RandomState((int(seed) + 77) % (2 ** 31))
        st["leaf_host"] = [int(r.randint(n // 2, n)) for n in new]
        st["leaf"] = torch.tensor(st["leaf_host"], dtype=torch.int32, device="cuda")
    if own:
        mp = st["mp"]
        if c["kind"] in ("turn", "append"):
            st["rotary"] = mp.MpRotary(rot_dim=c["rot"], layout=mp.MP_ROTARY_INTERLEAVED if c["interleaved"] else mp.MP_ROTARY_HALF, base=c["base"],
                                       scaling=mp.MP_ROTARY_BY_PARTS if c["factor"] > 1.0 else mp.MP_ROTARY_PLAIN, factor=c["factor"],
                                       original_len=8192, low=1.0, high=32.0, amplitude=st["amplitude"])
            st["q_norm"], st["k_norm"] = (mp.MpHeadNorm(st[w] if c["per_head"] else st[w][0], offset=c["offset"], eps=c["eps"]) for w in ("q_weight", "k_weight"))
        if c["kind"] != "turn":
            st["paged"] = mp.MpPagedKv(st["k_pages"], st["v_pages"], st["page_table"], st["kv_len"], st["q_start"])
        if c["kind"] == "attend":
            st["workspace"] = torch.empty(max(1, mp.mp_paged_workspace_bytes(T, Hq, Hkv, B, max(new))), dtype=torch.uint8, device="cuda")
    return st


def _prepare_reserve(c, seed, st):
    have, stay, come = _requests(c)
    B, page = c["B"], c["page"]
    columns = -(-(max(max(h, s + n) for h, s, n in zip(have, stay, come))) // page) + 2
    wanted = sum(-(-(s + n) // page) for s, n in zip(stay, come)) - sum(-(-h // page) for h in have)
    used = sum(-(-s // page) for s in stay)
    more = sum(-(-(s + n) // page) for s, n in zip(stay, come)) - used
    # enough for all, or (tight) for some three quarters of them once those that have ended have given theirs back
    spare = max(0, wanted - more // 4) if c["tight"] else max(0, wanted) + 16
    st["page_table"], free, n_pages = _page_table(c, have, columns, seed, spare)
    r = np.random.RandomState((int(seed) + 3) % (2 ** 31))
    st["free_pages"] = torch.full((n_pages,), -1, dtype=torch.int32)
    st["free_pages"][:len(free)] = torch.from_numpy(r.permutation(free).astype(np.int32))
    st["free_pages"] = st["free_pages"].cuda()
    for name, v in (("n_free", [len(free)]), ("kv_len", have), ("keep", stay), ("n_new", come), ("q_start", [0] * (B + 1)), ("granted", [0] * B)):
        st[name] = torch.tensor(v, dtype=torch.int32, device="cuda")
    rows = sum(come)
    st["sequence"], st["positions"] = (torch.full((rows,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    st["slots"] = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    if own:
        st["pool"] = st["mp"].MpPagePool(st["page_table"], st["kv_len"], st["q_start"], st["free_pages"], st["n_free"], page)
    return st


# ---------------------------------------------------------------------------------------- plain form
def _turned(x, positions, st):
    """x [..., heads, 128], in 32 bits, at positions [...]: the first `rot` dimensions turned."""
    c = st["case"]
    r, half = c["rot"], c["rot"] // 2
    a = positions.double()[..., None, None] * st["freqs"]
    cos, sin = (torch.cos(a) * st["amplitude"]).float(), (torch.sin(a) * st["amplitude"]).float()
    if c["interleaved"]:
        u, w = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([u * cos - w * sin, w * cos + u * sin], dim=-1).flatten(-2)
    else:
        u, w = x[..., :half], x[..., half:r]
        y = torch.cat([u * cos - w * sin, w * cos + u * sin], dim=-1)
    return torch.cat([y, x[..., r:]], dim=-1).to(torch.bfloat16)


def _normed(x, weight, c):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + c["eps"]) * (weight.float() + c["offset"])


def _rows(pages, table):
    """[n_pages, Hkv, page, 128] -> [B, Hkv, pages * page, 128]"""
    x = pages[table.long().clamp(min=0)]
    return x.transpose(1, 2).flatten(2, 3)


def _places(st):
    """Rows [B, N] of the sequences' new tokens (those of short sequences repeat others), and which are there."""
    starts = st["q_start"].long()
    n_new = starts[1:] - starts[:-1]
    i = torch.arange(max(st["new"]), device="cuda")
    return (starts[:-1, None] + i).clamp(max=st["T"] - 1), i < n_new[:, None], n_new


def _plain_plan(st):
    c = st["case"]
    rows, there, n_new = _places(st)
    B, N = rows.shape
    W = _words(c)
    p = torch.where(there, st["parents_at"][rows].long(), -1)
    i = torch.arange(N, device="cuda")
    reach = ((p[:, :, None] == i) | (i[:, None] == i)).float()
    for _ in range(max(1, math.ceil(math.log2(N)))):          # ancestors up to twice as far
        reach = (torch.matmul(reach, reach) > 0).float()
    bits = torch.zeros(B, N, W * 64, dtype=torch.int64, device="cuda")
    bits[:, :, :N] = reach.long()
    mask = (bits.view(B, N, W, 64) << torch.arange(64, device="cuda")).sum(dim=-1)
    positions = (st["kv_len"].long() - n_new)[:, None] + reach.sum(dim=-1).long() - 1
    return {"mask": mask[there], "positions": positions[there].int()}


def _bits(mask, rows, N):
    """The marked new tokens [B, N, N] of rows [B, N]."""
    m = mask[rows]
    return ((m[..., None] >> torch.arange(64, device="cuda")) & 1).flatten(-2)[..., :N] != 0


def _plain_attend(st):
    c = st["case"]
    B, Hq, Hkv, L, N = c["B"], c["Hq"], c["Hkv"], max(st["keys"]), max(st["new"])
    G = Hq // Hkv
    rows, there, n_new = _places(st)
    lens = st["kv_len"].long()
    older = lens - n_new
    q = st["q"][rows].view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D).float()
    K = _rows(st["k_pages"], st["page_table"])[:, :, :L].float()
    s = torch.matmul(q, K.transpose(2, 3)).mul_(SCALE).view(B, Hkv, N, G, L)
    del K
    j = torch.arange(L, device="cuda")
    bits = _bits(st["mask"], rows, N)
    seen = (j < older[:, None])[:, None].expand(B, N, L)
    in_tree = (j - older[:, None]).clamp(0, N - 1)[:, None].expand(B, N, L)
    seen = seen | ((j >= older[:, None]) & (j < lens[:, None]))[:, None] & bits.gather(2, in_tree)
    if c["window"]:                                             # the last ones of what each token would see
        seen = seen & (seen.flip(-1).int().cumsum(dim=-1).flip(-1) <= c["window"])
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    V = _rows(st["v_pages"], st["page_table"])[:, :, :L].float()
    o = torch.matmul(p.view(B, Hkv, N * G, L), V).view(B, Hkv, N, G, D) / l
    lse = (l.log() + m)[..., 0]
    out = o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)[there].to(torch.bfloat16)
    return {"out": out, "lse": lse.permute(0, 2, 1, 3).reshape(B, N, Hq)[there]}


def _plain_keep(st):
    c = st["case"]
    N, page = max(st["new"]), c["page"]
    starts = st["q_start"].long()
    older = st["kv_len"].long() - (starts[1:] - starts[:-1])
    bits = _bits(st["mask"], starts[:-1] + st["leaf"].long(), N)                # [B, N]
    rank = bits.long().cumsum(dim=-1) - 1
    b, j = bits.nonzero(as_tuple=True)
    src, dst = older[b] + j, older[b] + rank[b, j]
    from_page, to_page = st["page_table"][b, src // page].long(), st["page_table"][b, dst // page].long()
    for pages in (st["k_pages"], st["v_pages"]):
        pages[to_page, :, dst % page] = pages[from_page, :, src % page]
    return {"keep": (older + bits.sum(dim=-1)).int(), "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_reserve(st):
    P, table = st["case"]["page"], st["page_table"]
    B, S = table.shape
    n_pages, room = st["free_pages"].numel(), S * P
    e = torch.arange(S, device="cuda")
    have = st["kv_len"].long().clamp(0, room)
    stay = torch.minimum(st["keep"].long().clamp(min=0), have)
    had, left = (have + P - 1) // P, (stay + P - 1) // P
    # pages behind what stays go back
    goes = (e >= left[:, None]) & (e < had[:, None])
    back = (goes & (table >= 0) & (table < n_pages)).flatten()
    stack = torch.cat([st["free_pages"], st["free_pages"].new_zeros(1)])
    top = st["n_free"][0].long() + back.sum()
    at = st["n_free"][0].long() + back.long().cumsum(0) - 1
    stack.scatter_(0, torch.where(back, at, n_pages), table.flatten())
    table = torch.where(goes, -1, table)
    # tokens to come, as long as there are pages for them
    come = st["n_new"].long().clamp(min=0)
    fits = stay + come <= room
    need = torch.where(fits, (stay + come + P - 1) // P - left, 0)
    ok = fits & ((need == 0) | (need.cumsum(0) <= top))
    granted, take = torch.where(ok, come, 0), torch.where(ok, need, 0)
    upto = take.cumsum(0)
    rank = (upto - take)[:, None] + e - left[:, None]
    takes = (e >= left[:, None]) & (e < (left + take)[:, None])
    table = torch.where(takes, stack[(top - 1 - rank).clamp(0, n_pages)], table)
    total = upto[-1]
    place = torch.arange(n_pages, device="cuda")
    st["free_pages"].copy_(torch.where((place >= top - total) & (place < top), -1, stack[:n_pages]))
    st["n_free"].copy_((top - total).int())
    st["page_table"].copy_(table)
    st["kv_len"].copy_((stay + granted).int())
    q_start = torch.cat([granted.new_zeros(1), granted.cumsum(0)])
    st["q_start"].copy_(q_start.int())
    st["granted"].copy_(granted.int())
    # a step's rows
    r = torch.arange(st["slots"].numel(), device="cuda")
    seq = torch.searchsorted(q_start[1:], r, right=True)
    valid = seq < B
    seq = seq.clamp(max=B - 1)
    pos = st["kv_len"].long()[seq] - (q_start[seq + 1] - r)
    slot = table[seq, (pos // P).clamp(0, S - 1)].long() * P + pos % P
    st["sequence"].copy_(torch.where(valid, seq, -1).int())
    st["positions"].copy_(torch.where(valid, pos, -1).int())
    st["slots"].copy_(torch.where(valid, slot, -1))
    return _reserved(st)


def _reserved(st):
    return {k: st[k] for k in ("page_table", "kv_len", "q_start", "free_pages", "n_free", "granted", "sequence", "positions", "slots")}


def _plain(st):
    c = st["case"]
    if c["kind"] == "turn":
        x = _normed(st["q"], st["q_weight"], c)
        return {"out": _turned(x, st["positions"], st), "lookup": _turned(x, torch.full_like(st["positions"], LOOKUP_AT), st)}
    if c["kind"] == "append":
        seq = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), (st["q_start"][1:] - st["q_start"][:-1]).long(), output_size=st["T"])
        pos = st["positions"].long()
        page, slot = st["page_table"][seq, pos // c["page"]].long(), pos % c["page"]
        st["k_pages"][page, :, slot] = _turned(_normed(st["k"], st["k_weight"], c), st["positions"], st)
        st["v_pages"][page, :, slot] = st["v"]
        return {"q": _turned(_normed(st["q"], st["q_weight"], c), st["positions"], st), "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if c["kind"] == "reserve":
        return _plain_reserve(st)
    if c["kind"] == "plan":
        return _plain_plan(st)
    if c["kind"] == "attend":
        return _plain_attend(st)
    return _plain_keep(st)


# ---------------------------------------------------------------------------------------- the framework's calls
def _own(st):
    c = st["case"]
    if c["kind"] == "turn":
        out, lookup = st["rotary"].mp_norm_rotary(st["q_norm"], st["q"], st["positions"], lookup_position=LOOKUP_AT)
        return {"out": out, "lookup": lookup}
    if c["kind"] == "append":
        q = st["paged"].mp_paged_append_norm(st["k"], st["v"], rotary=st["rotary"], q=st["q"], q_norm=st["q_norm"], k_norm=st["k_norm"], positions=st["positions"])
        return {"q": q, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if c["kind"] == "reserve":
        st["pool"].mp_paged_reserve(n_new=st["n_new"], keep=st["keep"], granted=st["granted"], sequence=st["sequence"], positions=st["positions"], slots=st["slots"])
        return _reserved(st)
    if c["kind"] == "plan":
        mask, positions = st["paged"].mp_paged_tree_plan(st["parents_at"], mask_words=_words(c))
        return {"mask": mask, "positions": positions}
    if c["kind"] == "attend":
        lse = torch.empty(st["T"], c["Hq"], dtype=torch.float32, device="cuda")
        out = st["paged"].mp_paged_tree_attention(st["q"], st["mask"], max_new=max(st["new"]), window=c["window"], lse=lse, workspace=st["workspace"])
        return {"out": out, "lse": lse}
    keep = st["paged"].mp_paged_tree_keep(st["mask"], st["leaf"])
    return {"keep": keep, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------------------------------- in 64 bits
def _turned_exactly(x, positions, st):
    """The pairs as complex numbers, times e^(i angle)."""
    c = st["case"]
    r, half = c["rot"], c["rot"] // 2
    pairs = x[..., :r].unflatten(-1, (half, 2)) if c["interleaved"] else x[..., :r].unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = positions.double()[..., None, None] * st["freqs"]
    z = z * torch.polar(torch.full_like(angle, st["amplitude"]), angle)
    y = torch.view_as_real(z)
    y = y.flatten(-2) if c["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _normed_exactly(x, weight, c):
    x = x.double()
    return x / torch.sqrt((x.norm(dim=-1, keepdim=True) ** 2) / D + c["eps"]) * (weight.double() + c["offset"])


def _ancestors(parents, i):
    path = []
    while i >= 0:
        path.append(i)
        i = int(parents[i])
    return path[::-1]


def _sequence(st, name, b):
    """The pages of one sequence as [Hkv, keys, 128]."""
    page, n = st["case"]["page"], st["keys"][b]
    ids = st["page_table"][b, :-(-n // page)].long()
    return st[name][ids].permute(1, 0, 2, 3).reshape(st["case"]["Hkv"], -1, D)[:, :n]


def exact(c, seed):
    if c["kind"] in ("reserve", "plan"):
        return None                                             # whole numbers
    st = prepare(c, seed)
    B, Hq, Hkv = c["B"], c["Hq"], c["Hkv"]
    G = Hq // Hkv
    if c["kind"] == "turn":
        x = _normed_exactly(st["q"], st["q_weight"], c)
        return {"out": _turned_exactly(x, st["positions"], st), "lookup": _turned_exactly(x, torch.full_like(st["positions"], LOOKUP_AT), st)}
    first = [0]
    for n in st["new"]:
        first.append(first[-1] + n)
    if c["kind"] == "append":
        k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
        k = _turned_exactly(_normed_exactly(st["k"], st["k_weight"], c), st["positions"], st)
        for b in range(B):
            pos = torch.arange(st["keys"][b] - st["new"][b], st["keys"][b], device="cuda")
            page = st["page_table"][b].long()[torch.div(pos, c["page"], rounding_mode="floor")]
            k_pages[page, :, pos % c["page"]] = k[first[b]:first[b + 1]]
            v_pages[page, :, pos % c["page"]] = st["v"][first[b]:first[b + 1]].double()
        return {"q": _turned_exactly(_normed_exactly(st["q"], st["q_weight"], c), st["positions"], st), "k_pages": k_pages, "v_pages": v_pages}
    table = st["page_table"].cpu().numpy()
    if c["kind"] == "keep":
        k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
        for b in range(B):
            older = st["keys"][b] - st["new"][b]
            path = _ancestors(st["parents"][b], st["leaf_host"][b])
            src = [(table[b, (older + i) // c["page"]], (older + i) % c["page"]) for i in path]
            rows = [(k_pages[p, :, s].clone(), v_pages[p, :, s].clone()) for p, s in src]
            for i, (k, v) in enumerate(rows):
                p, s = table[b, (older + i) // c["page"]], (older + i) % c["page"]
                k_pages[p, :, s], v_pages[p, :, s] = k, v
        return {"keep": None, "k_pages": k_pages, "v_pages": v_pages}
    out = torch.empty(st["T"], Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["T"], Hq, dtype=torch.float64, device="cuda")
    for b in range(B):
        K, V = _sequence(st, "k_pages", b), _sequence(st, "v_pages", b)
        n, k = st["new"][b], st["keys"][b]
        older = k - n
        seen = torch.zeros(n, k, dtype=torch.bool)
        for i in range(n):
            path = _ancestors(st["parents"][b], i)
            if c["window"]:
                path = path[-c["window"]:]
            seen[i, max(0, older - (c["window"] - len(path))) if c["window"] else 0:older] = True
            seen[i, [older + a for a in path]] = True
        seen = seen.cuda()
        for h in range(Hkv):
            x = st["q"][first[b]:first[b + 1], h * G:(h + 1) * G].double().reshape(n * G, D)
            s = (x @ K[h].double().t().contiguous() * SCALE).view(n, G, k).masked_fill(~seen[:, None], -math.inf)
            lse[first[b]:first[b + 1], h * G:(h + 1) * G] = torch.logsumexp(s, dim=2)
            out[first[b]:first[b + 1], h * G:(h + 1) * G] = (torch.softmax(s, dim=2).view(n * G, k) @ V[h].double()).view(n, G, D)
    return {"out": out, "lse": lse}
