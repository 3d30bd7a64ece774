"""Plain forms in 64 bits of the calls on int8 codes, the error bounds that follow from the kernels' arithmetic, and strided operands for the tests.

Rounding: U = 2^-24 is half a unit in the last place of fp32, HALF[dtype] that of an output's type.  A sum of n terms formed by lanes of at most c terms each
and a tree is within (c + log2 n + 2) U of the sum of the magnitudes."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}  # spacing of the smallest numbers
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def generator(seed, *more):
    g = torch.Generator(device="cuda")
    return g.manual_seed(hash((seed,) + more) & 0x7FFFFFFFFFFF)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def codes_of(g, *shape):
    return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int16).to(torch.int8)


def placed(t, pad, offset, fill):
    """The values of a 2-D tensor in rows that are `pad` elements longer and start `offset` elements into memory; `fill` elsewhere."""
    rows, cols = t.shape
    whole = torch.full((rows * (cols + pad) + offset,), fill, dtype=t.dtype, device=t.device)
    view = whole[offset:].as_strided((rows, cols), (cols + pad, 1))
    view.copy_(t)
    return whole, view


def untouched(whole, view, fill):
    """Whether everything but the view still holds `fill`."""
    other = torch.ones_like(whole, dtype=torch.bool)
    other[view.storage_offset():].as_strided(view.shape, view.stride()).fill_(False)
    return bool((whole[other] == fill).all())


def sum_error(n):
    """Factor of U for a sum over a row of n: 8 to 32 values a lane in registers, more beyond 32768."""
    return 8 * max(4, math.ceil(n / 8192)) + math.log2(n + 1) + 4


def silu(x):
    return x * torch.sigmoid(x)


def assert_quantized(codes, scale, y, relative):
    """codes, scale against the rows y (64 bits), whose values the kernel has within `relative` of themselves and whose scale within `relative`."""
    top = y.abs().amax(dim=1)
    assert codes.dtype == torch.int8 and scale.dtype == torch.float32
    assert ((scale.double() - top / 127).abs() <= relative * top / 127 + 2.0 ** -149).all()
    zero = top == 0
    assert (codes[zero] == 0).all()
    want = torch.where(zero[:, None], 0.0, y * 127 / torch.where(zero, 1.0, top)[:, None])
    # half a code, and what the errors of the value and of the largest are in codes
    assert ((codes.double() - want).abs() <= 0.5 + 127 * 2 * relative).all()
    assert (codes.double().abs().amax(dim=1)[~zero] == 127).all()


def assert_near(got, want, error):
    """Every element within `error` (a tensor, for the arithmetic) and the rounding of the output's type."""
    slack = error * (1 + HALF[got.dtype]) + HALF[got.dtype] * want.abs() + LEAST[got.dtype]
    most = torch.finfo(got.dtype).max
    beyond = want.abs() > most * (1 + HALF[got.dtype]) + slack  # rounds to infinity
    assert (got[beyond] == torch.sign(want[beyond]) * math.inf).all()
    off = torch.where(beyond | (torch.isinf(got) & (want.abs() + slack > most)), 0.0, (got.double() - want).abs())
    assert (off <= slack).all(), (off / slack).max().item()


def moe(x, sx, logits, top, w1, s1, w2, s2):
    """Mixture-of-experts layer in 64 bits -> (out, error bound).  An activation whose code lies within 1e-3 of the middle between two may get either (fp32 has it within
  some 90 U of itself, twice that with the largest, times 127):
    the bound has the difference."""
    T, H = x.shape
    F = w2.shape[2]
    out = torch.zeros(T, H, dtype=torch.float64, device=x.device)
    error = torch.zeros_like(out)
    table = logits.double().cpu().tolist()
    for t in range(T):
        row = table[t]
        if any(v != v or v == math.inf for v in row):
            out[t] = math.nan
            continue
        best = sorted(range(len(row)), key=lambda e: (-row[e], e))[:top]
        if row[best[0]] == -math.inf:
            continue
        odds = [math.exp(row[e] - row[best[0]]) for e in best]
        for e, o in zip(best, odds):
            if o < 2.0 ** -149:
                continue
            p = o / sum(odds)
            u = (w1[e].double() @ x[t].double()) * sx[t].double() * s1[e].double()
            a = silu(u[:F]) * u[F:]
            largest = a.abs().max()
            if not torch.isfinite(largest):
                out[t] = math.nan
                continue
            v = torch.zeros_like(a) if largest == 0 else a * 127 / largest
            code = torch.round(v)
            open_ = ((v - torch.floor(v) - 0.5).abs() < 1e-3).double()
            W, scale = w2[e].double(), s2[e].double() * largest / 127
            out[t] += p * scale * (W @ code)
            error[t] += p * scale * (W.abs() @ open_ + 100 * U * (W @ code).abs())
    return out, error
