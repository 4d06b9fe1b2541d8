"""Trees of drafted tokens and pools of pages, written out step by step."""
import math

import torch

from tests.paged_util import BF16


def random_parents(n, seed, deep=0.5):
    """Of n tokens, each one's parent before it; the first, and now and then another, has none (-1)."""
    g = torch.Generator().manual_seed(seed)
    p = []
    for i in range(n):
        r = float(torch.rand(1, generator=g))
        p.append(-1 if i == 0 or r < 0.05 else i - 1 if r < deep else int(torch.randint(0, i, (1,), generator=g)))
    return p


def ancestors(parents, i):
    path = []
    while 0 <= i < len(parents):
        path.append(i)
        i = parents[i] if parents[i] < i else -1
    return path[::-1]


def words_of(marked, words):
    """64-bit words (as signed numbers) with the bits of `marked` set."""
    w = [0] * words
    for j in marked:
        if j < 64 * words:
            w[j // 64] |= 1 << (j % 64)
    return [x - (1 << 64) if x >> 63 else x for x in w]


def tree_attention(b, q, marked, window=0, scale=None):
    """`marked`: of every sequence, of every new token, the new ones it marks.  (out, lse, bound of out, bound of lse) in fp64, rows of no sequence NaN; bounds as in Batch.attention."""
    scale = scale or 1.0 / math.sqrt(128)
    T, Hq = q.shape[0], q.shape[1]
    G = Hq // b.Hkv
    out, obound = (torch.full((T, Hq, 128), math.nan, dtype=torch.float64, device="cuda") for _ in range(2))
    lse, lbound = (torch.full((T, Hq), math.nan, dtype=torch.float64, device="cuda") for _ in range(2))
    for s, (n, k) in enumerate(zip(b.new, b.lens)):
        if n == 0:
            continue
        older = k - n
        seen = torch.zeros(n, max(k, 0), dtype=torch.bool)
        for i in range(n):
            keys = list(range(max(older, 0))) + [older + j for j in sorted(marked[s][i]) if j < n]
            keys = [j for j in (keys[-window:] if window else keys) if j >= 0]
            seen[i, keys] = True
        seen = seen.cuda() & b.there(s)[None]
        rows = slice(b.starts[s], b.starts[s + 1])
        for h in range(Hq):
            K, V = b.keys[s][h // G].double(), b.values[s][h // G].double()
            x = q[rows, h].double()
            z = (x @ K.t().contiguous() * scale).masked_fill(~seen, -math.inf)
            m = z.amax(1, keepdim=True) if z.shape[1] else torch.full((n, 1), -math.inf, dtype=torch.float64, device="cuda")
            e = torch.exp(z - torch.where(m.isinf(), torch.zeros_like(m), m))
            l = e.sum(1, keepdim=True)
            w = torch.where(l > 0, e / l, torch.zeros_like(e))
            V = torch.where(seen.any(0)[:, None], V, torch.zeros_like(V))
            o, size = w @ V, w @ V.abs()
            d = 130 * 2.0 ** -24 * scale * (x.norm(dim=1, keepdim=True) * (K.norm(dim=1).max() if K.shape[0] else 0.0))
            n_keys = seen.sum(1, keepdim=True)
            out[rows, h] = o
            obound[rows, h] = BF16 * o.abs() + (BF16 + 2 * d + (n_keys + 64) * 2.0 ** -24) * size
            lse[rows, h] = (m + l.log())[:, 0]
            lbound[rows, h] = (d + (n_keys + 64) * 2.0 ** -24 + 2.0 ** -22 * (m.abs() + 1))[:, 0].nan_to_num(posinf=0.0)
    return out, lse, obound, lbound


class Pool:
    """Lists of what mp_paged_reserve changes, and what it does to them, entry by entry."""

    def __init__(self, page, columns, n_pages, seqs, seed=0, have=None):
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(n_pages, generator=g).tolist()
        self.page, self.columns, self.n_pages = page, columns, n_pages
        self.kv_len = list(have) if have else [0] * seqs
        self.table = [[-1] * columns for _ in range(seqs)]
        for b, k in enumerate(self.kv_len):
            for e in range(-(-k // page)):
                self.table[b][e] = order.pop()
        self.stack = order + [-1] * (n_pages - len(order))
        self.n_free = len(order)
        self.q_start = [0] * (seqs + 1)

    def step(self, come, keep=None, rows=0):
        P, room = self.page, self.columns * self.page
        up = lambda x: -(-x // P)      # noqa: E731
        have = [min(max(k, 0), room) for k in self.kv_len]
        stay = [min(max(k, 0), h) for k, h in zip(have if keep is None else keep, have)]
        for b, (h, s) in enumerate(zip(have, stay)):
            for e in range(up(s), up(h)):
                if 0 <= self.table[b][e] < self.n_pages and self.n_free < self.n_pages:
                    self.stack[self.n_free] = self.table[b][e]
                    self.n_free += 1
                self.table[b][e] = -1
        granted, short = [], False
        for b, (s, n) in enumerate(zip(stay, come)):
            n = max(n, 0)
            more = up(s + n) - up(s)
            if s + n > room:
                n = more = 0
            short = short or more > self.n_free
            if more and short:
                n = more = 0
            for e in range(up(s), up(s) + more):
                self.n_free -= 1
                self.table[b][e], self.stack[self.n_free] = self.stack[self.n_free], -1
            granted.append(n)
            self.kv_len[b] = s + n
            self.q_start[b + 1] = self.q_start[b] + n
        seq, pos, slots = [], [], []
        for b, n in enumerate(granted):
            for p in range(self.kv_len[b] - n, self.kv_len[b]):
                seq.append(b)
                pos.append(p)
                e = self.table[b][p // P]
                slots.append(e * P + p % P if 0 <= e < self.n_pages else -1)
        fill = [-1] * max(0, rows - len(seq))
        return granted, (seq + fill)[:rows], (pos + fill)[:rows], (slots + fill)[:rows]
