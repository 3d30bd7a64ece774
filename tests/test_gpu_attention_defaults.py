"""How a call of attention over the cache is split where the caller does not say how many new tokens a sequence has."""
import pytest
import torch

from attention_testlib import Paged, attention, heads_of
from int8_testlib import assert_near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,fresh,planned", [([300] * 40, [1] * 40, 1), ([300] * 40, [1] * 30 + [0] * 10, 1), ([300] * 40, [30] + [0] * 39, 1), ([300] * 3, [1, 2, 1], 4),
                                                   ([900], [900], 900), ([50], [1], 1)])
def test_without_most_new(seed, lengths, fresh, planned, monkeypatch):
    """No more tokens than sequences: as for one token each.  Otherwise one sequence could have them all."""
    import paper_1609_07061_amd as q

    p = Paged(seed, lengths, fresh, 1, 64, 16)
    x = heads_of(seed, p.tokens, 4, 64, torch.bfloat16)
    asked = []
    need = q.qnn_cache_attention_workspace_bytes
    monkeypatch.setattr(q, "qnn_cache_attention_workspace_bytes", lambda *a: asked.append(a) or need(*a))
    got = q.qnn_cache_attention(x, *p.args, longest=max(lengths))
    assert [a[5] for a in asked] == [planned]
    want, error, written = attention(p, x, 0.125)
    assert_near(got[written], want[written], error[written])
    assert torch.equal(got, q.qnn_cache_attention(x, *p.args, most_new=planned, longest=max(lengths)))
