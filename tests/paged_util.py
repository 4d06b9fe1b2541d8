"""A paged cache with sequences in it, and the operators over it written out in 64 bits."""
import math

import torch

BF16 = 2.0 ** -8       # half a step of bf16, relative


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def turned(x, positions, freqs, interleaved, amplitude=1.0):
    """x [tokens, heads, 128] (any type) -> fp64, from the formula pair by pair."""
    x = x.double()
    r = 2 * freqs.numel()
    a = positions.double().view(-1, 1, 1) * freqs.to(x.device).double()
    cos, sin = a.cos() * amplitude, a.sin() * amplitude
    i = torch.arange(r // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    y = x.clone()
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    return y


def turn_bound(x, want, freqs, interleaved, amplitude=1.0):
    """One rounding to bf16; cosine, sine (2^-23 of one each, their argument as much) and two products and a sum in fp32 of the pair's elements."""
    r = 2 * freqs.numel()
    size = x.double().abs()
    pair = size[..., :r]
    pair = pair + (pair.unflatten(-1, (r // 2, 2)).flip(-1).flatten(-2) if interleaved else pair.roll(r // 2, dims=-1))
    extra = torch.zeros_like(size)
    extra[..., :r] = pair * abs(amplitude) * 2.0 ** -20
    return BF16 * want.abs() + extra


class Batch:
    """Sequences of `new` tokens behind len - new older ones.  What no sequence holds of the cache is NaN, unused entries name no page.
    `columns`: of the page table, at least."""

    def __init__(self, new, lens, Hkv, page, seed=1, pad_front=0, pad_back=0, spare=2, stale=math.nan, scale=1.0, columns=0):
        g = gen(seed)
        self.new, self.lens, self.Hkv, self.page = list(new), list(lens), Hkv, page
        n = [max(0, -(-k // page)) for k in lens]
        width = max(max(n + [1]) + 1, columns)
        self.n_pages = sum(n) + spare
        order = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        table = torch.full((len(lens), width), -1, dtype=torch.int32)
        table[:, -1] = self.n_pages + 7
        at = 0
        for b, k in enumerate(n):
            table[b, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
            at += k
        shape = (self.n_pages, Hkv, page, 128)
        self.K, self.V = (torch.full(shape, stale, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.table = table.cuda()
        starts = [pad_front]
        for k in new:
            starts.append(starts[-1] + k)
        self.starts, self.T = starts, starts[-1] + pad_back
        self.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.keys, self.values = [], []
        for b, k in enumerate(self.lens):
            k = max(k, 0)
            self.keys.append((scale * torch.randn(Hkv, k, 128, generator=g, device="cuda")).to(torch.bfloat16))
            self.values.append(torch.randn(Hkv, k, 128, generator=g, device="cuda").to(torch.bfloat16))
        self.write()

    def write(self):
        for b, k in enumerate(self.lens):
            if k > 0:
                page, slot = self.where(b, torch.arange(k, device="cuda"))
                self.K[page, :, slot] = self.keys[b].transpose(0, 1)
                self.V[page, :, slot] = self.values[b].transpose(0, 1)

    def where(self, b, positions):
        return self.table[b].long()[positions // self.page], positions % self.page

    def paged(self):
        from paper_2506_13059_amd import binding as mp
        return mp.MpPagedKv(self.K, self.V, self.table, self.kv_len, self.q_start)

    def positions(self, b):
        return torch.arange(self.lens[b] - self.new[b], self.lens[b], device="cuda")

    def there(self, b):
        """Which keys of a sequence lie on a page."""
        k = max(self.lens[b], 0)
        e = self.table[b].long()[torch.arange(k, device="cuda") // self.page]
        return (e >= 0) & (e < self.n_pages)

    def attention(self, q, window=0, scale=None):
        """(out, lse, bound of out, bound of lse) in fp64, rows of no sequence NaN.

        Bounds: with d the error of a logit (fp32 sums of 128 products, and its product with the scale), a probability is off by
        2 d and by its rounding to bf16, sums of n terms in fp32 by n 2^-24 at most, and the result is rounded to bf16 once."""
        scale = scale or 1.0 / math.sqrt(128)
        T, Hq = q.shape[0], q.shape[1]
        G = Hq // self.Hkv
        out, obound = (torch.full((T, Hq, 128), math.nan, dtype=torch.float64, device="cuda") for _ in range(2))
        lse, lbound = (torch.full((T, Hq), math.nan, dtype=torch.float64, device="cuda") for _ in range(2))
        for b in range(len(self.lens)):
            p = self.positions(b)[:, None]
            j = torch.arange(max(self.lens[b], 0), device="cuda")[None]
            seen = (j <= p) & self.there(b)[None]
            if window:
                seen = seen & (p - j < window)
            rows = slice(self.starts[b], self.starts[b + 1])
            for h in range(Hq):
                K, V = self.keys[b][h // G].double(), self.values[b][h // G].double()
                x = q[rows, h].double()
                s = (x @ K.t().contiguous() * scale).masked_fill(~seen, -math.inf)
                m = s.amax(1, keepdim=True) if s.shape[1] else torch.full((x.shape[0], 1), -math.inf, dtype=torch.float64, device="cuda")
                e = torch.exp(s - torch.where(m.isinf(), torch.zeros_like(m), m))
                l = e.sum(1, keepdim=True)
                w = torch.where(l > 0, e / l, torch.zeros_like(e))
                o = w @ torch.where(seen.any(0)[:, None], V, torch.zeros_like(V))
                size = w @ torch.where(seen.any(0)[:, None], V.abs(), torch.zeros_like(V))
                d = 130 * 2.0 ** -24 * scale * (x.norm(dim=1, keepdim=True) * (K.norm(dim=1).max() if K.shape[0] else 0.0))
                n = seen.sum(1, keepdim=True)
                out[rows, h] = o
                obound[rows, h] = BF16 * o.abs() + (BF16 + 2 * d + (n + 64) * 2.0 ** -24) * size
                lse[rows, h] = (m + l.log())[:, 0]
                lbound[rows, h] = (d + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * (m.abs() + 1))[:, 0].nan_to_num(posinf=0.0)
        return out, lse, obound, lbound


def check(got, want, bound, label):
    got = got.double()
    bad = ~((got - want).abs() <= bound) & ~((got == want) & want.isinf())
    assert not bad.any(), f"{label}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}, bound {bound[bad][0]}"
