"""Performance cases of the operators that carry a prompt, and the tokens behind it, through a paged cache.

Rotary positions (`mp_rotary`), appending to the cache with the rotation on the way (`mp_paged_append`), attention of new tokens over
it (`mp_paged_attention`), and the rows of its sequences in order, with the keys turned to one position, as the k-means build takes
them (`mp_paged_gather`).

Where `own` is false, `run` computes the same in elementary torch operations in 32 bits (angles in 64), rounded once at the end.

Keys have four channels far from zero in every head, the same way for all tokens, as key caches have them; queries are drawn so that
logits have a standard deviation of about two; values are N(0, 1).  Pages are handed out in random order.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
MOST_PAIRS = 2.7e8 * 32      # (query, key, head) triples: no drawn case has more than the largest listed one
MOST_ROWS = 16 * 8 * 80000   # key rows (times two: and value rows) of a cache


# ---------------------------------------------------------------------------------------- cases
def _case(name, kind, B, Hq, Hkv, new, context, **more):
    base = dict(name=name, kind=kind, B=B, Hq=Hq, Hkv=Hkv, new=new, context=context, ragged=False, page=16, window=0, mixed=False,
                rot=128, interleaved=False, base=1e6, factor=1.0, lookup=False)
    base.update(more)
    return base


def listed():
    return [
        # a decode step of sixteen sequences: queries at their own positions and at the one that centroids are scored at
        _case("rotary_tokens_b16", "rotary", 16, 32, 8, 1, 131072, ragged=True, lookup=True),
        # a prompt's queries, taken from the rows of a fused projection; adjacent pairs of half of the head, frequencies scaled by parts
        _case("rotary_prompt_8k_g5", "rotary", 1, 40, 8, 8191, 8191, rot=64, interleaved=True, base=1e4, factor=4.0),
        # one token each of sixteen sequences joins the cache: the smallest append, every step of a server
        _case("append_tokens_b16", "append", 16, 32, 8, 1, 32768, ragged=True),
        # five prompts' tokens of odd numbers go to pages of 64, frequencies scaled for a long context
        _case("append_prompts_b5_g5", "append", 5, 40, 8, 4099, 20000, ragged=True, page=64, factor=8.0),
        # one token over 4096 keys: the smallest attention call, a single user
        _case("attend_token_4k_b1", "attend", 1, 32, 8, 1, 4096),
        # one token each of sixteen sequences of up to 128K: the largest of decode's calls
        _case("attend_tokens_128k_b16", "attend", 16, 32, 8, 1, 131072, ragged=True, page=64),
        # a few drafted tokens a sequence, checked together; groups of eight query heads
        _case("attend_drafts_30k_b8_g8", "attend", 8, 64, 8, 5, 30011, ragged=True),
        # a server's step: tokens of fifteen sequences and a piece of another's prompt, with a window
        _case("attend_mixed_16k_b16_window", "attend", 16, 32, 8, 333, 16384, ragged=True, mixed=True, window=4096),
        # a whole prompt, heads of a 14B model (groups of five)
        _case("attend_prompt_8k_g5", "attend", 1, 40, 8, 8192, 8192, page=64),
        # the last piece of a prompt of 128K: the largest call
        _case("attend_chunk_2k_at_128k", "attend", 1, 32, 8, 2048, 131072, page=64),
        # one prompt's rows for the k-means build, with lookup keys
        _case("gather_32k_b1", "gather", 1, 32, 8, 1, 32768, lookup=True),
        # four prompts of 64K, large pages, lookup keys
        _case("gather_64k_b4_g5", "gather", 4, 40, 8, 1, 65521, page=256, lookup=True, factor=4.0, rot=96),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotary", "append", "attend", "attend", "attend", "gather"])
        Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
        c = dict(kind=kind, B=_log_int(rng, 1, 33), Hq=Hkv * G, Hkv=Hkv, ragged=rng.random() < 0.7, page=rng.choice([16, 32, 64, 128, 256]),
                 rot=rng.choice([32, 64, 96, 128]), interleaved=rng.random() < 0.4, base=rng.choice([1e4, 5e5, 1e6]),
                 factor=rng.choice([1.0, 4.0, 8.0]), lookup=kind == "gather" or (kind == "rotary" and rng.random() < 0.5),
                 new=1, window=0, mixed=False)
        c["context"] = _log_int(rng, 17, 131072)
        if kind in ("rotary", "append"):
            c["new"] = _log_int(rng, 1, 8192)
        elif kind == "attend":
            how = rng.choice(["token", "drafts", "chunk"])
            c["new"] = 1 if how == "token" else rng.randint(2, 9) if how == "drafts" else _log_int(rng, 10, 8192)
            c["window"] = rng.choice([0, 0, 0, 1023, 4096])
            c["mixed"] = how == "chunk" and rng.random() < 0.3
        c["new"] = min(c["new"], c["context"])
        rows = c["B"] * c["Hkv"] * c["context"]
        pairs = c["B"] * c["Hq"] * c["new"] * c["context"]      # of the plain form, which pads
        tokens = c["B"] * c["new"] * (c["Hq"] + 2 * c["Hkv"])
        if rows <= MOST_ROWS and (kind != "attend" or pairs <= MOST_PAIRS) and tokens <= 5 * 4099 * 56:
            return c


# ---------------------------------------------------------------------------------------- sizes of a case
def _lengths(c):
    """(new tokens, keys with them) of every sequence."""
    rng = random.Random(c["B"] * 1000003 + c["context"] * 31 + c["new"])
    new, keys = [], []
    for b in range(c["B"]):
        full = b == 0 or not c["ragged"]
        n = c["new"] if full else 1 if c["mixed"] else c["new"] if c["new"] < 16 else rng.randint(max(1, c["new"] // 2), c["new"])
        k = c["context"] if full else int(c["context"] * math.exp(rng.uniform(math.log(0.125), 0.0)))
        new.append(n)
        keys.append(max(n, k))
    return new, keys


def _visible(c):
    """(query, key) pairs that are attended, and keys that some query attends, per head."""
    pairs = rows = 0
    for n, k in zip(*_lengths(c)):
        for_each = np.arange(k - n + 1, k + 1, dtype=np.int64)
        if c["window"]:
            for_each = np.minimum(for_each, c["window"])
        pairs += int(for_each.sum())
        rows += min(k, n - 1 + c["window"]) if c["window"] else k
    return pairs, rows


def work(c):
    new, keys = _lengths(c)
    T, Hq, Hkv, row = sum(new), c["Hq"], c["Hkv"], D * 2
    if c["kind"] == "rotary":
        return {"bytes": T * Hq * row * (3 if c["lookup"] else 2) + 4 * T, "flops": T * Hq * c["rot"] * 3 * (2 if c["lookup"] else 1)}
    if c["kind"] == "append":
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * row, "flops": T * (Hq + Hkv) * c["rot"] * 3}
    if c["kind"] == "attend":
        pairs, rows = _visible(c)
        return {"bytes": rows * Hkv * 2 * row + T * Hq * (2 * row + 4), "flops": 4 * D * Hq * pairs}
    n = c["context"]
    return {"bytes": sum(keys) * Hkv * 2 * row + c["B"] * Hkv * n * 3 * row, "flops": sum(keys) * Hkv * c["rot"] * 3}


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


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)
    new, keys = _lengths(c)
    B, Hq, Hkv, page, T = c["B"], c["Hq"], c["Hkv"], c["page"], sum(new)
    st = dict(case=c, new=new, keys=keys, T=T, freqs=torch.from_numpy(_frequencies(c)).cuda(), amplitude=_amplitude(c))
    starts = np.concatenate([[0], np.cumsum(new)])
    st["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    st["kv_len"] = torch.tensor(keys, dtype=torch.int32, device="cuda")
    pos = np.concatenate([np.arange(k - n, k) for n, k in zip(new, keys)])
    st["positions"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
    if c["kind"] in ("rotary", "append"):
        # the rows of a fused projection: queries, keys, values of a token behind one another
        st["qkv"] = _keys((T, Hq + 2 * Hkv, D), 1, g)
        st["q"], st["k"], st["v"] = st["qkv"][:, :Hq], st["qkv"][:, Hq:Hq + Hkv], st["qkv"][:, Hq + Hkv:]
    elif c["kind"] == "attend":
        st["q"] = (2.0 * torch.randn(T, Hq, D, generator=g, device="cuda")).to(torch.bfloat16)
    if c["kind"] != "rotary":
        need = [-(-k // page) for k in keys]
        n_pages = sum(need) + 3
        table = np.full((B, max(need)), -1, dtype=np.int32)
        order = np.random.RandomState(int(seed) % (2 ** 31)).permutation(n_pages)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        st["page_table"] = torch.from_numpy(table).cuda()
        st["k_pages"] = _keys((n_pages, Hkv, page, D), 1, g)
        st["v_pages"] = torch.randn(n_pages, Hkv, page, D, generator=g, device="cuda", dtype=torch.bfloat16)
    if own:
        from paper_2506_13059_amd import binding as mp
        st["mp"] = mp
        st["rotary"] = mp.MpRotary(rot_dim=c["rot"], layout=mp.MP_ROTARY_INTERLEAVED if c["interleaved"] else mp.MP_ROTARY_HALF, base=c["base"],
                                   scaling=mp.MP_ROTARY_BY_PARTS if c["factor"] > 1.0 else mp.MP_ROTARY_PLAIN, factor=c["factor"],
                                   original_len=8192, low=1.0, high=32.0, amplitude=st["amplitude"])
        if c["kind"] != "rotary":
            st["paged"] = mp.MpPagedKv(st["k_pages"], st["v_pages"], st["page_table"], st["kv_len"], st["q_start"])
        if c["kind"] == "attend":
            st["workspace"] = torch.empty(max(1, mp.mp_paged_workspace_bytes(T, Hq, Hkv, B, max(new))), dtype=torch.uint8, device="cuda")
    return st


LOOKUP_AT = 4096      # the position that lookup keys and queries are turned to


# ---------------------------------------------------------------------------------------- plain form
def _turned(x, positions, st, amplitude):
    """x [..., heads, 128] at positions [...]: the first `rot` dimensions turned, in 32 bits."""
    c = st["case"]
    r, half = c["rot"], c["rot"] // 2
    a = positions.double()[..., None, None] * st["freqs"]
    cos, sin = (torch.cos(a) * amplitude).float(), (torch.sin(a) * amplitude).float()
    x = x.float()
    if c["interleaved"]:
        u, w = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([u * cos - w * sin, w * cos + u * sin], dim=-1).flatten(-2)
    else:
        u, w = x[..., :half], x[..., half:r]
        y = torch.cat([u * cos - w * sin, w * cos + u * sin], dim=-1)
    return torch.cat([y, x[..., r:]], dim=-1).to(torch.bfloat16)


def _rows(pages, table):
    """[n_pages, Hkv, page, 128] -> [B, Hkv, pages * page, 128]"""
    x = pages[table.long().clamp(min=0)]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(st):
    c = st["case"]
    B, Hq, Hkv, L, N = c["B"], c["Hq"], c["Hkv"], max(st["keys"]), max(st["new"])
    G = Hq // Hkv
    starts, lens = st["q_start"].long(), st["kv_len"].long()
    n_new = starts[1:] - starts[:-1]
    i = torch.arange(N, device="cuda")
    rows = (starts[:-1, None] + i).clamp(max=st["T"] - 1)                      # [B, N], those of short sequences repeat others
    at = lens[:, None] - n_new[:, None] + i                                    # positions
    q = st["q"][rows].view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D).float()
    K = _rows(st["k_pages"], st["page_table"])[:, :, :L].float()
    s = torch.matmul(q, K.transpose(2, 3)).mul_(SCALE).view(B, Hkv, N, G, L)
    del K
    j = torch.arange(L, device="cuda")
    seen = (j <= at[..., None]) & (j < lens[:, None, None])
    if c["window"]:
        seen &= j > at[..., None] - c["window"]
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    V = _rows(st["v_pages"], st["page_table"])[:, :, :L].float()
    o = torch.matmul(p.view(B, Hkv, N * G, L), V).view(B, Hkv, N, G, D) / l
    lse = (l.log() + m)[..., 0]
    there = i < n_new[:, None]
    out = o.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)[there].to(torch.bfloat16)
    return {"out": out, "lse": lse.permute(0, 2, 1, 3).reshape(B, N, Hq)[there]}


def _plain(st):
    c = st["case"]
    if c["kind"] == "rotary":
        r = {"out": _turned(st["q"], st["positions"], st, st["amplitude"])}
        if c["lookup"]:
            r["lookup"] = _turned(st["q"], torch.full_like(st["positions"], LOOKUP_AT), st, st["amplitude"])
        return r
    if c["kind"] == "append":
        seq = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), (st["q_start"][1:] - st["q_start"][:-1]).long(), output_size=st["T"])
        pos = st["positions"].long()
        page, slot = st["page_table"][seq, pos // c["page"]].long(), pos % c["page"]
        st["k_pages"][page, :, slot] = _turned(st["k"], st["positions"], st, st["amplitude"])
        st["v_pages"][page, :, slot] = st["v"]
        return {"q": _turned(st["q"], st["positions"], st, st["amplitude"]), "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if c["kind"] == "attend":
        return _plain_attend(st)
    n = c["context"]
    k, v = _rows(st["k_pages"], st["page_table"])[:, :, :n], _rows(st["v_pages"], st["page_table"])[:, :, :n]
    at = torch.arange(n, device="cuda", dtype=torch.int32)
    there = (at < st["kv_len"][:, None])[:, None, :, None]
    k, v = k * there, v * there
    turned = _turned(k.transpose(1, 2), (LOOKUP_AT - at).expand(c["B"], n), st, 1.0).transpose(1, 2).contiguous()
    return {"k": k, "v": v, "k_lookup": turned}


# ---------------------------------------------------------------------------------------- the framework's calls
def _own(st):
    c = st["case"]
    if c["kind"] == "rotary":
        if c["lookup"]:
            out, lookup = st["rotary"].mp_rotary(st["q"], st["positions"], lookup_position=LOOKUP_AT)
            return {"out": out, "lookup": lookup}
        return {"out": st["rotary"].mp_rotary(st["q"], st["positions"])}
    if c["kind"] == "append":
        q = st["paged"].mp_paged_append(st["k"], st["v"], rotary=st["rotary"], q=st["q"])
        return {"q": q, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if c["kind"] == "attend":
        lse = torch.empty(st["T"], c["Hq"], dtype=torch.float32, device="cuda")
        out = st["paged"].mp_paged_attention(st["q"], max_new=max(st["new"]), window=c["window"], lse=lse, workspace=st["workspace"])
        return {"out": out, "lse": lse}
    k, v, k_lookup = st["paged"].mp_paged_gather(c["context"], rotary=st["rotary"], lookup_position=LOOKUP_AT)
    return {"k": k, "v": v, "k_lookup": k_lookup}


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------------------------------- in 64 bits
def _turned_exactly(x, positions, st, amplitude):
    """The pairs as complex numbers, times e^(i angle)."""
    c = st["case"]
    r, half = c["rot"], c["rot"] // 2
    x = x.double()
    pairs = x[..., :r].unflatten(-1, (half, 2)) if c["interleaved"] else x[..., :r].unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = positions.double()[..., None, None] * st["freqs"]
    z = z * torch.polar(torch.full_like(angle, amplitude), angle)
    y = torch.view_as_real(z)
    y = y.flatten(-2) if c["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _sequence(st, name, b):
    """The pages of one sequence as [Hkv, keys, 128]."""
    page, n = st["case"]["page"], st["keys"][b]
    ids = st["page_table"][b, :-(-n // page)].long()
    return st[name][ids].permute(1, 0, 2, 3).reshape(st["case"]["Hkv"], -1, D)[:, :n]


def exact(c, seed):
    pairs, _ = _visible(c)
    if c["kind"] == "attend" and pairs * c["Hq"] > MOST_PAIRS * 1.1:
        return None
    st = prepare(c, seed)
    B, Hq, Hkv = c["B"], c["Hq"], c["Hkv"]
    G = Hq // Hkv
    if c["kind"] == "rotary":
        r = {"out": _turned_exactly(st["q"], st["positions"], st, st["amplitude"])}
        if c["lookup"]:
            r["lookup"] = _turned_exactly(st["q"], torch.full_like(st["positions"], LOOKUP_AT), st, st["amplitude"])
        return r
    first = [0]
    for n in st["new"]:
        first.append(first[-1] + n)
    if c["kind"] == "append":
        k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
        k = _turned_exactly(st["k"], st["positions"], st, st["amplitude"])
        for b in range(B):
            pos = torch.arange(st["keys"][b] - st["new"][b], st["keys"][b], device="cuda")
            page = st["page_table"][b].long()[torch.div(pos, c["page"], rounding_mode="floor")]
            k_pages[page, :, pos % c["page"]] = k[first[b]:first[b + 1]]
            v_pages[page, :, pos % c["page"]] = st["v"][first[b]:first[b + 1]].double()
        return {"q": _turned_exactly(st["q"], st["positions"], st, st["amplitude"]), "k_pages": k_pages, "v_pages": v_pages}
    if c["kind"] == "attend":
        out = torch.empty(st["T"], Hq, D, dtype=torch.float64, device="cuda")
        lse = torch.empty(st["T"], Hq, dtype=torch.float64, device="cuda")
        for b in range(B):
            K, V = _sequence(st, "k_pages", b), _sequence(st, "v_pages", b)
            n, k = st["new"][b], st["keys"][b]
            for i0 in range(0, n, 1024):
                i1 = min(n, i0 + 1024)
                p = torch.arange(k - n + i0, k - n + i1, device="cuda")[:, None]
                j = torch.arange(k, device="cuda")[None]
                seen = j <= p
                if c["window"]:
                    seen = seen & (p - j < c["window"])
                for h in range(Hq):
                    q = st["q"][first[b] + i0:first[b] + i1, h].double()
                    s = (q @ K[h // G].double().t().contiguous() * SCALE).masked_fill(~seen, -math.inf)
                    lse[first[b] + i0:first[b] + i1, h] = torch.logsumexp(s, dim=1)
                    out[first[b] + i0:first[b] + i1, h] = torch.softmax(s, dim=1) @ V[h // G].double()
        return {"out": out, "lse": lse}
    n = c["context"]
    k, v = (torch.zeros(B, Hkv, n, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        k[b, :, :st["keys"][b]] = _sequence(st, "k_pages", b).double()
        v[b, :, :st["keys"][b]] = _sequence(st, "v_pages", b).double()
    back = (LOOKUP_AT - torch.arange(n, device="cuda"))[:, None].expand(n, Hkv)
    turned = torch.stack([_turned_exactly(k[b].transpose(0, 1), back[:, 0], st, 1.0).transpose(0, 1) for b in range(B)])
    return {"k": k, "v": v, "k_lookup": turned}
