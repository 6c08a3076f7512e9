"""A batch over a shared prefix in a paged cache, and the definitions of rotation and attention in 64 bits."""
from __future__ import annotations

import math

import torch

# half a step of the type's grid, relative (bf16 has 8 significant bits, fp16 11, fp32 24)
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def rotated(x, positions, theta, axis_pairs, interleaved, amplitude=1.0, inverse=False):
    """x [heads, tokens, dim] float64; positions [axes, tokens]; theta [pairs] radians a position (float64)."""
    rot = 2 * len(theta)
    axis = torch.repeat_interleave(torch.arange(len(axis_pairs)), torch.tensor(axis_pairs))
    angle = positions.double()[axis].t() * theta                       # [tokens, pairs]
    c, s = angle.cos() * amplitude, angle.sin() * amplitude * (-1 if inverse else 1)
    y = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rotation_tolerance(x, rot, interleaved, amplitude, dtype):
    """What a rotation in fp32 may be off, element by element: the angle is 32 bits of a turn, taken to fp32 (error below
    pi 2^-24 + 2 pi 2^-32), sine and cosine carry two roundings more, the products and their sum three: below 8 * 2^-24 of
    |a| + |b|; then one rounding to the tensor's type (and half its smallest number)."""
    y = torch.zeros_like(x)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = y[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(amplitude)
    return y * (8 * 2.0 ** -24), UNIT[dtype] if dtype != torch.float32 else 0.0


class Batch:
    """Sequences with `new` new tokens and `own` own keys each over `prefix` shared keys, in a cache whose unused slots and
    pages hold NaN."""

    def __init__(self, new, own, prefix, kv_heads=2, group=1, dim=128, page=16, dtype=torch.bfloat16, token_major=False, seed=0,
                 q_scale=1.0, spare_tokens=0, spare_pages=3, rise=0.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.own, self.prefix, self.page, self.dim, self.dtype = new, own, prefix, page, dim, dtype
        self.kv_heads, self.group, self.heads = kv_heads, group, kv_heads * group
        need = [-(-n // page) for n in own]
        shared = -(-prefix // page)
        self.n_pages = shared + sum(need) + spare_pages
        order = torch.randperm(self.n_pages, generator=g)
        shape = (self.n_pages, page, kv_heads, dim) if token_major else (self.n_pages, kv_heads, page, dim)
        view = (lambda t: t.transpose(1, 2)) if token_major else (lambda t: t)
        self.k, self.v = (view(torch.full(shape, math.nan, dtype=dtype)) for _ in range(2))
        self.prefix_pages = order[:shared].to(torch.int32)
        wide = max(need + [0])
        self.table = torch.full((len(new), wide), -7, dtype=torch.int32)            # entries behind a sequence's pages are not read
        at = shared
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        for keys, pages in [(prefix, self.prefix_pages)] + [(n, self.table[b]) for b, n in enumerate(own)]:
            ramp = 1.0 + rise * torch.arange(keys)[:, None] / max(keys, 1)
            self.put(self.k, pages, torch.randn(kv_heads, keys, dim, generator=g) * ramp)
            self.put(self.v, pages, torch.randn(kv_heads, keys, dim, generator=g))
        self.seq_start = torch.tensor([0] + new).cumsum(0).to(torch.int32)
        self.kv_len = torch.tensor(own, dtype=torch.int32)
        self.tokens = sum(new) + spare_tokens
        self.q = (torch.randn(self.tokens, self.heads, dim, generator=g) * q_scale).to(dtype).transpose(0, 1)

    def put(self, cache, pages, x):
        n = x.shape[1]
        for i in range(0, n, self.page):
            m = min(self.page, n - i)
            cache[int(pages[i // self.page]), :, :m] = x[:, i:i + m].to(self.dtype)

    def get(self, cache, pages, n):
        if n == 0:
            return cache.new_zeros((self.kv_heads, 0, self.dim)).double()
        x = cache[pages[:-(-n // self.page)].long()]                                # [pages, heads, page, dim]
        return x.transpose(0, 1).reshape(self.kv_heads, -1, self.dim)[:, :n].double()

    def cuda(self):
        for name in ("k", "v", "prefix_pages", "table", "seq_start", "kv_len", "q"):
            setattr(self, name, getattr(self, name).cuda())
        return self

    def expected(self, causal, scale=None):
        """o, lse in 64 bits, and what o and lse may be off (all on the CPU; call it before cuda())."""
        scale = scale or 1.0 / math.sqrt(self.dim)
        o = torch.zeros((self.heads, self.tokens, self.dim), dtype=torch.float64)
        lse = torch.full((self.heads, self.tokens), -math.inf, dtype=torch.float64)
        o_tol, lse_tol = torch.zeros_like(o), torch.zeros_like(lse)
        kp, vp = self.get(self.k, self.prefix_pages, self.prefix), self.get(self.v, self.prefix_pages, self.prefix)
        unit = UNIT[self.dtype]
        for b, (n, have) in enumerate(zip(self.new, self.own)):
            t = int(self.seq_start[b])
            k = torch.cat([kp, self.get(self.k, self.table[b], have)], 1)
            v = torch.cat([vp, self.get(self.v, self.table[b], have)], 1)
            for i in range(n):
                see = self.prefix + (max(0, have - n + i + 1) if causal else have)
                if see == 0:
                    continue
                for h in range(self.heads):
                    kh, vh, q = k[h // self.group, :see], v[h // self.group, :see], self.q[h, t + i].double()
                    x = (kh @ q) * scale
                    w = torch.softmax(x, 0)
                    o[h, t + i] = w @ vh
                    lse[h, t + i] = torch.logsumexp(x, 0)
                    # a score is a sum of dim products in fp32 (dim roundings of partial sums at most), its exponential is taken
                    # by an instruction good to 2^-22 of an argument rounded once; sums are fp32
                    size = float((kh.abs() @ q.abs()).max()) * scale
                    e = (self.dim + 2) * 2.0 ** -24 * size + 2.0 ** -20
                    lse_tol[h, t + i] = e + 2.0 ** -22 * abs(float(lse[h, t + i]))
                    # p is rounded to the type for the second product, the result once more
                    mean = w @ vh.abs()
                    o_tol[h, t + i] = mean * (unit + 2 * e) + o[h, t + i].abs() * unit + 2.0 ** -24
        return o, lse, o_tol, lse_tol
