"""Plain forms in 64 bits of the calls on heads and the paged cache, with the error bounds that follow from the kernels' arithmetic, and the inputs of their tests.

U = 2^-24 is half a unit in the last place of fp32, as in int8_testlib."""
from __future__ import annotations

import math

import torch

from int8_testlib import U, generator, normal

NORM = 14  # U of r = 1 / sqrt(mean + eps): a sum of 16 squares a lane and 4 joins, halved by the root, and quotient, root, quotient
TURN = 6   # U of a cosine or sine: the angle in fp32 (pi / 4), polynomial, and its sums


def heads_of(seed, tokens, heads, D, dtype, scale=1.0):
    g = generator(seed, tokens, heads, D)
    return (normal(g, tokens, heads, D) * torch.exp(0.5 * normal(g, heads, D)) * scale).to(dtype)


def strided(t, dtype=None, fill=float("nan")):
    """The values of a [tokens][heads][D] tensor as a part of longer rows, heads apart from each other, at an odd address."""
    T, H, D = t.shape
    whole = torch.full((T * (H * (D + 3) + 5) + 1,), fill, dtype=dtype or t.dtype, device=t.device)
    view = whole[1:].as_strided((T, H, D), (H * (D + 3) + 5, D + 3, 1))
    view.copy_(t)
    return whole, view


def untouched(whole, view, fill):
    other = torch.ones_like(whole, dtype=torch.bool)
    other[view.storage_offset():].as_strided(view.shape, view.stride()).fill_(False)
    left = whole[other]
    return bool(torch.isnan(left).all() if fill != fill else (left == fill).all())


class Rotation:
    def __init__(self, seed, tokens, D, pairs=None, axes=1, neighbours=False, most=5000):
        g = generator(seed, tokens, D, axes)
        self.pairs = D // 2 if pairs is None else pairs
        self.positions = torch.randint(-3, most, (axes, tokens), generator=g, device="cuda", dtype=torch.int32)
        self.freq = 10000.0 ** (-torch.arange(self.pairs, device="cuda", dtype=torch.float64) / max(self.pairs, 1))
        self.axis = None if axes == 1 else torch.randint(0, axes, (self.pairs,), generator=g, device="cuda", dtype=torch.int32)
        self.neighbours = neighbours

    @property
    def args(self):
        return self.positions, self.freq, self.axis, self.neighbours

    def angles(self):
        p = self.positions.double()
        rows = p[:1].expand(self.pairs, -1) if self.axis is None else p[self.axis.long()]
        return (rows.t() * self.freq)[:, None]  # [tokens][1][pairs]

    def parts(self, y):
        """(first, second) of the pairs, and the rest."""
        n = 2 * self.pairs
        if self.neighbours:
            return y[..., 0:n:2], y[..., 1:n:2], y[..., n:]
        return y[..., :self.pairs], y[..., self.pairs:n], y[..., n:]

    def join(self, a, b, rest):
        both = torch.stack([a, b], dim=-1).flatten(-2) if self.neighbours else torch.cat([a, b], dim=-1)
        return torch.cat([both, rest], dim=-1)

    def turn(self, y, error, sign):
        """y turned (64 bits), and the bound of its error from that of y."""
        a, b, rest = self.parts(y)
        ea, eb, er = self.parts(error)
        angle = self.angles()
        c, s = torch.cos(angle), sign * torch.sin(angle)
        size = (a.abs() + b.abs()) * (TURN * U + angle.abs() * 2.0 ** -51) + 2 * U * (a.abs() + b.abs())
        both = (ea.square() + eb.square()).sqrt() * math.sqrt(2)
        return self.join(a * c - b * s, b * c + a * s, rest), self.join(size + both, size + both, er)


def norm_rotate(x, gamma, eps, rotation):
    """(values, bound of their error before the output's rounding)."""
    h = x.double()
    if gamma is None:
        return rotation.turn(h, torch.zeros_like(h), 1)
    n = h / torch.sqrt(h.square().mean(dim=-1, keepdim=True) + eps) * gamma.double()
    return rotation.turn(n, n.abs() * (NORM + 2) * U, 1)


def norm_rotate_backward(grad, x, gamma, eps, rotation):
    """(gradient, its error; gamma's gradient, its error)."""
    g, e = rotation.turn(grad.double(), torch.zeros_like(grad, dtype=torch.float64), -1)
    if gamma is None:
        return g, e, None, None
    h, w = x.double(), gamma.double()
    D, n = h.shape[-1], h.shape[0] * h.shape[1]
    r = 1 / torch.sqrt(h.square().mean(dim=-1, keepdim=True) + eps)
    mean = lambda t: t.mean(dim=-1, keepdim=True)
    out = r * (w * g - h * r * r * mean(w * g * h))
    error = r * (w.abs() * e + (w * g).abs() * (NORM + 4) * U)
    error += r * h.abs() * r * r * (mean((w * h).abs() * e) + mean((w * g * h).abs()) * (3 * NORM + 24 + 6) * U)
    # a thread adds at most every item that it could have, then 32 threads and the parts' tree
    chain = math.ceil(n / 32) + 32 + 48
    sums = (g * h * r).sum(dim=(0, 1))
    wrong = ((h * r).abs() * e).sum(dim=(0, 1)) + (g * h * r).abs().sum(dim=(0, 1)) * (NORM + 2 + chain) * U
    return out, error, sums, wrong


# ----------------------------------------------------------------------------------------------------------- the cache
class Paged:
    """A cache of random codes and the tables of sequences whose pages lie in any order.  lengths and fresh: of every sequence."""

    def __init__(self, seed, lengths, fresh, heads, D, page, spare=2, before=0, behind=0):
        g = generator(seed, sum(lengths), heads, D, page)
        self.n, self.fresh, self.heads, self.D, self.page = list(lengths), list(fresh), heads, D, page
        need = [-(-n // page) for n in lengths]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).tolist()
        self.table = torch.full((len(need), max(need + [1]) + 1), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(need):
            for i in range(n):
                self.table[b, i] = order.pop()
        starts = [before]
        for f in fresh:
            starts.append(starts[-1] + f)
        self.tokens = starts[-1] + behind
        self.first = starts
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        self.starts, self.lengths = ints(starts), ints(list(lengths))
        codes = lambda: torch.randint(-127, 128, (pages, heads, page, D), generator=g, device="cuda", dtype=torch.int16).to(torch.int8)
        scale = lambda: torch.rand(pages, heads, page, generator=g, device="cuda") * 0.03 + 0.005
        self.cache = (codes(), scale(), codes(), scale())

    @property
    def args(self):
        return self.cache, self.table, self.starts, self.lengths

    def places(self, b):
        """(page, offset, whether there is one) of every token of a sequence."""
        at = torch.arange(self.n[b], device="cuda")
        number = at // self.page
        inside = number < self.table.shape[1]
        page = torch.where(inside, self.table[b].long()[number.clamp(max=self.table.shape[1] - 1)], -1)
        there = (page >= 0) & (page < self.cache[0].shape[0])
        return page.clamp(0, self.cache[0].shape[0] - 1), at % self.page, there


def attention(p: Paged, q, scale, cap=0.0, slopes=None, tree=None):
    """(out in 64 bits, bound of its error before the output's rounding, the rows that the call writes)."""
    T, H, D = q.shape
    group = H // p.heads
    out = torch.zeros(T, H, D, dtype=torch.float64, device="cuda")
    error, written = torch.zeros_like(out), torch.zeros(T, dtype=torch.bool, device="cuda")
    parts = 2 if q.dtype == torch.float32 else 1
    masks = None if tree is None else [m & (1 << 64) - 1 for m in tree.tolist()]
    for b, (n, m) in enumerate(zip(p.n, p.fresh)):
        rows = slice(p.first[b], p.first[b] + m)
        written[rows] = True
        if n == 0 or m == 0:
            continue
        page, off, there = p.places(b)
        key, base = torch.arange(n, device="cuda"), n - m
        place_k = key
        if tree is None:
            place_q = base + torch.arange(m, device="cuda")
            sees = key[None] <= place_q[:, None]
        else:
            mine = masks[rows]
            seen = [[j < base or (j - base < 64 and bool(x >> (j - base) & 1)) for j in range(n)] for x in mine]
            sees = torch.tensor(seen, device="cuda")
            place_q = torch.tensor([base - 1 + bin(x).count("1") for x in mine], device="cuda")
            place_k = torch.cat([key[:base], place_q]) if base >= 0 else place_q[-base:]
        sees = sees & there[None]
        for h in range(H):
            c = h // group
            k = p.cache[0][page, c, off].double() * p.cache[1][page, c, off].double()[:, None]
            bs = p.cache[3][page, c, off].double()
            v = p.cache[2][page, c, off].double() * bs[:, None]
            k, v, bs = (torch.where(there.view(-1, *[1] * (t.dim() - 1)), t, 0.0) for t in (k, v, bs))
            x = q[rows, h].double()
            s = scale * (x @ k.t())
            size = abs(scale) * (x.abs() @ k.abs().t())
            d = (D + 20) * U * size  # what the score is off by
            if cap:
                s = cap * torch.tanh(s / cap)
                d = d + 12 * U * s.abs()
            if slopes is not None:
                bias = slopes[h].double() * (place_q[:, None] - place_k[None]).double()
                s, d = s - bias, d + 4 * U * bias.abs()
            s = torch.where(sees, s, -math.inf)
            top = s.amax(dim=1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            # exponents: product with log2(e), difference from R (which follows s + log2(b), log2(b) within 100 here), exp2
            d = d + 4 * U * (torch.where(sees, s.abs(), 0.0) + top.abs() + 100) + 4 * U
            e = torch.where(sees, torch.exp(s - top), 0.0)
            total = e.sum(dim=1, keepdim=True)
            w = torch.where(total > 0, e / total, 0.0)
            off_by = torch.where(sees, d, 0.0).amax(dim=1, keepdim=True)
            seen_v = torch.where(torch.isnan(v) & ~sees.any(dim=0)[:, None], 0.0, v)
            poisoned = (sees.double() @ torch.isnan(seen_v).any(dim=1).double()[:, None]) > 0
            clean = torch.nan_to_num(seen_v)
            y, most = w @ clean, w @ clean.abs()
            out[rows, h] = torch.where(poisoned | torch.isnan(s).any(dim=1, keepdim=True), math.nan, y)
            half = 2.0 ** -11 if parts == 1 else 2.0 ** -22
            least = n * 2.0 ** -33 * 127 * (w * torch.nan_to_num(bs)[None]).amax(dim=1, keepdim=True)
            error[rows, h] = most * (2 * off_by + half + (n / 8 + 64) * U) + least
    return out, error, written
