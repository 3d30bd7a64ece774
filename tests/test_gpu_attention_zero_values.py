"""Attention over tokens whose values are all zero (their scale is 0, as the call that appends writes it), against the definition in 64 bits: such tokens weigh like any other
and add nothing, however far their scores are from those of the tokens around them."""
import math

import pytest
import torch

from attention_testlib import Paged, attention, heads_of
from int8_testlib import U, assert_near, generator, normal

pytestmark = pytest.mark.gpu
N, HEADS, GROUP, D = 1500, 2, 4, 64
NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# What a weight 2^(t - R) b in float16 is off by, half of its least step, for every token: R lies 7 or more below the largest t + log2(max(b, 2^-96)), and the sum below the line is at least
# 2^(t - R) of that token, so that up to 2^-25 2^-7 2^-96 of a code is lost where tokens of zeros outweigh all others by as much as that.
FLOOR = N * 127 * 2.0 ** (-25 - 7 - 96)
WHICH = {"all": lambda i: i >= 0, "first": lambda i: i < N // 2, "last": lambda i: i >= N // 2, "steps": lambda i: i // 32 % 2 == 0, "tiles": lambda i: i // 64 % 2 == 1,
         "all but one": lambda i: i != 700}


def _scored(p, b, scores, values, scale):
    """Gives the tokens of sequence b these scores [n][heads] for a query of ones, and values this scale [n][heads]; where that is 0, codes are 0 too."""
    page, off, _ = p.places(b)
    p.cache[0][page, :, off] = torch.sign(scores).to(torch.int8)[..., None].expand(-1, -1, p.D)
    p.cache[1][page, :, off] = scores.abs() / (p.D * scale)
    p.cache[3][page, :, off] = values
    p.cache[2][page, :, off] *= (values != 0).to(torch.int8)[..., None]


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh", [1, 40, 400])  # few rows, more, and those of the kernel for many
@pytest.mark.parametrize("kind", ["plain", "cap", "slopes"])
@pytest.mark.parametrize("which", WHICH)
def test_scores_apart(seed, which, kind, fresh, type):
    """Scores from -180 to 180, so that weights without the values' scales are beyond fp32 from where a zero token was met first."""
    import paper_1609_07061_amd as q

    g = generator(seed, fresh)
    p = Paged(seed, [N], [fresh], HEADS, D, 16)
    at = torch.arange(N, device="cuda")
    zero = WHICH[which](at)
    zero = torch.stack([zero, zero if which == "all" else ~zero], dim=1)  # (the other head the other way round)
    scores = normal(g, N, HEADS) * 60
    scores[:, 1] = torch.where(zero[:, 1], (at - N / 2) * 0.2, normal(g, N))  # rising with the place, past 14 in every step of some rows
    if fresh > 1:
        scores[:, 1] = scores[:, 1].flip(0)
    _scored(p, 0, scores, torch.where(zero, 0.0, 0.01 + 0.02 * torch.rand(N, HEADS, generator=g, device="cuda")), 0.125)
    x = torch.ones(fresh, HEADS * GROUP, D, device="cuda", dtype=NAMES[type])
    x[:, 1::2] *= 0.5
    x[:, 2::4] *= -1
    options = {"cap": dict(cap=60.0), "slopes": dict(slopes=2.0 ** -torch.arange(8, device="cuda", dtype=torch.float32))}.get(kind, {})
    want, error, _ = attention(p, x, 0.125, **options)
    if which == "all":
        assert (want[:, :GROUP] == 0).all()
    for longest in (1, N):  # one part, and several
        assert_near(q.qnn_cache_attention(x, *p.args, 0.125, **options, most_new=fresh, longest=longest), want, error + FLOOR)


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh", [1, 400])
@pytest.mark.parametrize("size", [1e-25, 1e-3, 1e4, 1e9])
def test_beside_values_of_any_size(seed, size, fresh, type):
    """Zero tokens in steps of their own, from 20 below to 20 above the others' scores: they count in the sum whatever the others' scale is, across waves, parts and steps."""
    import paper_1609_07061_amd as q

    g = generator(seed, fresh, 5)
    p = Paged(seed, [N], [fresh], HEADS, D, 16)
    at = torch.arange(N, device="cuda")
    zero = (at // 64 % 2 == 0)[:, None].expand(-1, HEADS)
    scores = normal(g, N, HEADS)
    scores[:, 0] += torch.where(zero[:, 0], -1.0, 0.0)
    scores[:, 1] += torch.where(zero[:, 1], 20.0 - at * 40.0 / N, 0.0)
    _scored(p, 0, scores, torch.where(zero, 0.0, size * (0.5 + torch.rand(N, HEADS, generator=g, device="cuda"))), 0.125)
    x = torch.ones(fresh, HEADS * GROUP, D, device="cuda", dtype=NAMES[type])
    x[:, 1::2] *= 0.5
    if type == "f16" and size > 1:
        p.cache[2].zero_()  # (values beyond the type: zeros under these scales)
    want, error, _ = attention(p, x, 0.125)
    for longest in (1, N):
        assert_near(q.qnn_cache_attention(x, *p.args, 0.125, most_new=fresh, longest=longest), want, error + FLOOR)


@pytest.mark.parametrize("fresh", [1, 100])
def test_millions_of_zero_tokens(seed, fresh):
    """2.2 million tokens of zeros in one part, met before the one that has values: their number counts."""
    import paper_1609_07061_amd as q

    n, D, page, H = 2200000, 16, 2000, 8
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache = q.qnn_new_cache(n // page, 1, page, D)
    table = torch.arange(n // page, dtype=torch.int32, device="cuda")[None]
    at = (0, 5) if fresh > 1 else (n // page - 1, page - 1)  # (the last that its kernel meets, or nearly)
    cache[0][at[0], 0, at[1]] = 1
    cache[2][at[0], 0, at[1]] = torch.arange(1, D + 1, device="cuda").to(torch.int8)
    cache[3][at[0], 0, at[1]] = 0.5
    x = torch.ones(fresh, H, D, device="cuda")
    v = 0.5 * torch.arange(1, D + 1, device="cuda", dtype=torch.float64)
    for score in (math.log(n), 150.0):
        cache[1][at[0], 0, at[1]] = score / (D * 0.25)
        got = q.qnn_cache_attention(x, cache, table, ints([0, fresh]), ints([n]), 0.25, most_new=fresh, longest=1)
        s = cache[1][at[0], 0, at[1]].double() * D * 0.25
        others = (n - fresh + torch.arange(fresh, device="cuda", dtype=torch.float64))[:, None, None]  # seen beside it
        want = (v / (1 + others * torch.exp(-s))).expand(fresh, H, D)
        # the score within 4 U of itself, exponents of some 110 + |score| within 2 U, weights in two halves; the count is a sum of equal terms, whose error grows like a chain's of
        # n / 128 steps at most
        assert_near(got, want, want * (2 * U * (6 * (s + 110) + n / 128) + 2.0 ** -21))
