"""Queries that are not finite: NaN where they see anything, zeros where their masks and pages leave nothing, on either kernel."""
import math

import pytest
import torch

from attention_testlib import Paged, heads_of

pytestmark = pytest.mark.gpu
NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh", [1, 40, 400])  # few rows, more, and those of the kernel for many
@pytest.mark.parametrize("kind", ["plain", "cap", "slopes"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_queries(seed, bad, kind, fresh, type):
    import paper_1609_07061_amd as q

    p = Paged(seed, [500, 70], [fresh, 1], 2, 64, 16)
    p.table[0, :] = -1  # the first sequence has no pages ..
    x = heads_of(seed, p.tokens, 8, 64, NAMES[type])
    options = {"cap": dict(cap=30.0), "slopes": dict(slopes=torch.rand(8, device="cuda"))}.get(kind, {})
    call = lambda: q.qnn_cache_attention(x, *p.args, None, **options, most_new=fresh, longest=500)
    want = call().clone()
    assert (want[:fresh] == 0).all()
    x[0, 1, 5] = x[fresh - 1, 6, 63] = bad
    assert torch.equal(call(), want)
    p.table[0, 20] = 0  # .. then one in its middle, before all new tokens or among them
    x[0, 1, 5] = x[fresh - 1, 6, 63] = 0.5
    want = call().clone()
    x[0, 1, 5] = x[fresh - 1, 6, 63] = bad
    got = call()
    sees_first = 500 - fresh >= 20 * 16
    assert torch.isnan(got[fresh - 1, 6]).all() and (torch.isnan(got[0, 1]).all() if sees_first else (got[0, 1] == 0).all())
    got[fresh - 1, 6], got[0, 1] = want[fresh - 1, 6], want[0, 1]
    assert torch.equal(got, want)
    # masks of trees that leave nothing: their own, and a sequence of drafted tokens only
    p.table[1, :5] = torch.arange(5, device="cuda", dtype=torch.int32)
    if fresh == 40:
        p.table[0, :] = -1
        p.table[0, 31] = 1  # (tokens 496 .. 511: the last four of the drafted ones)
        tree = torch.zeros(p.tokens, dtype=torch.int64, device="cuda")
        tree[fresh - 1] = 1 << 39
        got = q.qnn_cache_attention(x, *p.args, None, **options, tree=tree, most_new=fresh, longest=500)
        assert (got[0] == 0).all() and torch.isnan(got[fresh - 1, 6]).all()
