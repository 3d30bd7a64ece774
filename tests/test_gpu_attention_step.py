"""The calls of the attention half together, as a block makes them: norm to codes, product, cache, attention, codes, product."""
import math
import os
import sys

import pytest
import torch

from attention_testlib import Paged, Rotation, attention, heads_of, norm_rotate
from int8_testlib import TYPES, U, assert_near, generator, normal

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EPS = 1e-6


class _Sequences:
    """Pages of several sequences, handed out as they grow."""

    def __init__(self, q, sequences, heads, D, page, room):
        per = -(-room // page)
        self.heads, self.D, self.page = heads, D, page
        self.cache = q.qnn_new_cache(sequences * per, heads, page, D)
        order = torch.randperm(sequences * per, generator=generator(1), device="cuda").to(torch.int32)
        self.table = order.view(sequences, per)
        self.n = [0] * sequences

    def step(self, fresh):
        self.fresh = fresh
        self.n = [a + b for a, b in zip(self.n, fresh)]
        self.first = [0]
        for f in fresh:
            self.first.append(self.first[-1] + f)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        self.starts, self.lengths = ints(self.first), ints(self.n)
        return self.cache, self.table, self.starts, self.lengths

    def places(self, b):
        at = torch.arange(self.n[b], device="cuda")
        return self.table[b].long()[at // self.page], at % self.page, torch.ones_like(at, dtype=torch.bool)


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_then_tokens(seed, dtype):
    """Prompts, single tokens and more of a prompt after each other: every step against the definition over what the cache holds, and the cache against one that
    got all tokens at once."""
    import paper_1609_07061_amd as q

    B, Hq, Hk, D, page = 3, 8, 2, 64, 16
    total = [70, 45, 90]
    qkv = [heads_of(seed + b, n, Hq + 2 * Hk, D, dtype) for b, n in enumerate(total)]
    gamma_q, gamma_k = ((1 + 0.2 * normal(generator(seed, i), D)).to(dtype) for i in range(2))
    freq = 10000.0 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) / (D // 2))
    one, many = _Sequences(q, B, Hk, D, page, 100), _Sequences(q, B, Hk, D, page, 100)

    def run(s, fresh):
        before = list(s.n)
        args = s.step(fresh)
        rows = torch.cat([x[a:a + f] for x, a, f in zip(qkv, before, fresh)])
        positions = torch.cat([torch.arange(a, a + f, device="cuda", dtype=torch.int32) for a, f in zip(before, fresh)])
        x, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]
        turned = q.qnn_cache_append(*args, k, v, gamma_k, EPS, positions, freq, q=x, gamma_q=gamma_q)
        out = q.qnn_cache_attention(turned, *args, most_new=max(fresh), longest=max(s.n))
        rotation = Rotation(seed, rows.shape[0], D)
        rotation.positions, rotation.freq = positions[None], freq
        assert_near(turned, *norm_rotate(x, gamma_q, EPS, rotation))
        want, error, written = attention(s, turned, D ** -0.5)
        assert written.all()
        assert_near(out, want, error)
        return [out[a:a + f] for a, f in zip(s.first, fresh)]

    whole = run(one, total)
    pieces = [[] for _ in range(B)]
    for fresh in ([40, 1, 33], [1, 1, 1], [1, 0, 20], [0, 40, 36], [28, 3, 0]):
        for got, part in zip(pieces, run(many, fresh)):
            got.append(part)
    assert many.n == one.n
    for b in range(B):
        (pa, oa, _), (pb, ob, _) = one.places(b), many.places(b)
        for s, t in zip(one.cache, many.cache):
            assert torch.equal(s[pa, :, oa], t[pb, :, ob])
        # the same queries over the same codes, split otherwise: twice the bound of either
        want, error, _ = attention(one, q.qnn_qk_norm_rotate(torch.cat(qkv)[:, :Hq], torch.cat(qkv)[:, :0], gamma_q, None, EPS, torch.cat([torch.arange(
            n, device="cuda", dtype=torch.int32) for n in total]), freq)[0], D ** -0.5)
        rows = slice(one.first[b], one.first[b + 1])
        assert_near(torch.cat(pieces[b]), want[rows], error[rows])
        assert_near(whole[b], want[rows], error[rows])


def test_into_the_output_product(seed):
    """The attention's result as codes into the output product."""
    import paper_1609_07061_amd as q

    g = generator(seed, 4)
    mixed = normal(g, 50, 8, 64).to(torch.bfloat16)
    w = torch.randint(-127, 128, (200, 512), generator=g, device="cuda", dtype=torch.int16).to(torch.int8)
    sw = torch.rand(200, generator=g, device="cuda") * 1e-3
    codes, scale = q.qnn_rows_quant(mixed.view(50, 512))
    y = q.qnn_int8_gemm(codes, scale, w, sw, dtype=torch.float32)
    want = (codes.double() @ w.double().t()) * scale.double()[:, None] * sw.double()
    assert_near(y, want, 4 * U * want.abs())
    # half a code at most from the values themselves
    true = mixed.view(50, 512).double() @ (w.double() * sw.double()[:, None]).t()
    assert ((y.double() - true).abs() <= (0.5 + 1e-5) * scale.double()[:, None] * (w.double().abs() * sw.double()[:, None]).sum(dim=1) + 1e-5).all()


def test_a_block_trains(seed):
    """Norm and rotation with their gradient around an attention in torch: the chain's gradients against those that torch has of the formulas."""
    import paper_1609_07061_amd as q

    T, Hq, Hk, D = 40, 4, 2, 32
    rotation = Rotation(seed, T, D)
    x, k, v = (heads_of(seed + i, T, H, D, torch.float32) for i, H in enumerate((Hq, Hk, Hk)))
    gq, gk = (1 + 0.2 * normal(generator(seed, i), D) for i in range(2))
    causal = torch.ones(T, T, dtype=torch.bool, device="cuda").tril()

    def mix(a, b):  # [T][H][D]
        b, c = (t.repeat_interleave(Hq // Hk, dim=1) for t in (b, v.to(a.dtype)))
        s = (a[:, None] * b[None]).sum(dim=3) / math.sqrt(D)  # [T][T][H]
        p = torch.softmax(torch.where(causal[..., None], s, -math.inf), dim=1)
        return (p[..., None] * c[None]).sum(dim=1)

    a, b = q.qnn_qk_norm_rotate(x, k, gq, gk, EPS, *rotation.args)
    a, b = a.requires_grad_(), b.requires_grad_()
    out = mix(a, b)
    up = normal(generator(seed, 9), *out.shape)
    out.backward(up)
    dx, dk, dgq, dgk = q.qnn_qk_norm_rotate_backward(a.grad, b.grad, x, k, gq, gk, EPS, *rotation.args)
    leaves = [t.double().requires_grad_() for t in (x, k, gq, gk)]
    angle = rotation.angles()
    c, s = torch.cos(angle), torch.sin(angle)

    def formula(h, w):
        n = h / torch.sqrt(h.square().mean(dim=-1, keepdim=True) + EPS) * w
        p, r, _ = rotation.parts(n)
        return torch.cat([p * c - r * s, r * c + p * s], dim=-1)

    mix(formula(leaves[0], leaves[2]), formula(leaves[1], leaves[3])).backward(up.double())
    for got, leaf in zip((dx, dk, dgq, dgk), leaves):
        # fp32 throughout, 335 U of the largest: values turned and turned back are off by some 30 U each, scores by 100, and what remains averages over 40 keys
        assert ((got.double() - leaf.grad).abs() <= 2e-5 * leaf.grad.abs().max()).all()


def test_given_buffers_and_new_ones(seed):
    """The binding's short way, for calls that bring all their buffers, and its general one: the same bits."""
    import paper_1609_07061_amd as q

    T, Hq, Hk, D = 21, 6, 2, 48
    p = Paged(seed, [30, 50], [20, 1], Hk, D, 16)
    rotation = Rotation(seed, T, D, 16, 2)
    x, k, v = (heads_of(seed + i, T, H, D, torch.bfloat16) for i, H in enumerate((Hq, Hk, Hk)))
    gq, gk = ((1 + 0.2 * normal(generator(seed, i), D)).to(torch.bfloat16) for i in range(2))
    new = lambda t: torch.full_like(t, 7)
    byte = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")

    def same(a, b):
        assert all(torch.equal(s, t) for s, t in zip(a, b, strict=True))

    same(q.qnn_qk_norm_rotate(x, k, gq, gk, EPS, *rotation.args, new(x), new(k)), q.qnn_qk_norm_rotate(x, k, gq, gk, EPS, *rotation.args))
    sums = [torch.full((D,), 7.0, device="cuda") for _ in range(2)]
    ws = byte(q.qnn_qk_norm_rotate_backward_workspace_bytes(T, Hq, Hk, D))
    same(q.qnn_qk_norm_rotate_backward(x, v, x, k, gq, gk, EPS, *rotation.args, new(x), new(k), *sums, ws), q.qnn_qk_norm_rotate_backward(x, v, x, k, gq, gk, EPS, *rotation.args))
    kept = [t.clone() for t in p.cache]
    short = q.qnn_cache_append(*p.args, k, v, gk, EPS, *rotation.args, x, gq, new(x))
    other = q.qnn_cache_append(tuple(kept), *p.args[1:], k, v, gk, EPS, *rotation.args, x, gq)
    same([short, *p.cache], [other, *kept])
    slopes = torch.rand(Hq, device="cuda")
    tree = torch.full((T,), 5, dtype=torch.int64, device="cuda")
    for options in (dict(), dict(cap=5.0, slopes=slopes), dict(tree=tree)):
        ws = byte(q.qnn_cache_attention_workspace_bytes(T, 2, Hq, Hk, D, 20, 50))
        same([q.qnn_cache_attention(x, *p.args, 0.2, **options, most_new=20, longest=50, out=new(x), workspace=ws)],
             [q.qnn_cache_attention(x, *p.args, 0.2, **options, most_new=20, longest=50)])
    rows = x.view(T, Hq * D)
    same(q.qnn_rows_quant(rows, new(rows).to(torch.int8), torch.empty(T, device="cuda")), q.qnn_rows_quant(rows))


def test_two_streams_at_once(seed):
    """Calls on two streams, each with buffers of its own: what each gives alone."""
    import paper_1609_07061_amd as q

    p = Paged(seed, [900, 3000], [1, 1], 2, 128, 16)
    xs = [heads_of(seed + i, 2, 8, 128, torch.bfloat16) for i in range(2)]
    want = [q.qnn_cache_attention(x, *p.args, most_new=1, longest=3000).clone() for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [[], []]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(q.qnn_cache_attention(xs[i], *p.args, most_new=1, longest=3000))
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for got, w in zip(outs, want) for o in got)


def test_example():
    sys.path.insert(0, ROOT)
    from examples import int8_attention as e

    got, want = e.serve()
    assert torch.isfinite(want).all() and torch.equal(got, want)
    tree, alone = e.check_drafts()
    # the same sums in another order, rounded to bf16, then to codes of which one in some hundred may differ
    assert torch.isfinite(tree).all() and (tree.float() - alone.float()).abs().max() <= 0.02 * alone.float().abs().max()
