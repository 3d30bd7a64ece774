"""The workspace of attention over the cache: one that is made for the most serves all calls."""
import pytest
import torch

from test_int8_refusals import SHAPE  # noqa: F401  (the package is built)


@pytest.mark.parametrize("D", [16, 64, 80, 128, 256])
def test_never_less_for_more(D):
    """More tokens or longer sequences need no less, and the numbers of sequences and of new tokens change nothing."""
    import paper_1609_07061_amd as q

    size = q.qnn_cache_attention_workspace_bytes
    longest = [1, 100, 128, 129, 1000, 5000, 8192, 100000, 1 << 31, 1 << 40]
    tokens = [1, 2, 3, 7, 16, 40, 64, 65, 200, 1000, 2048, 8192, 1 << 20]
    for heads_q, heads in ((1, 1), (8, 2), (32, 8), (32, 1), (64, 64)):
        before = [0] * len(longest)
        for t in tokens:
            row = [size(t, 1, heads_q, heads, D, t, n) for n in longest]
            assert row == sorted(row) and all(a >= b for a, b in zip(row, before))
            for sequences in (1, 3, 64, t):
                for most_new in {1, max(t // sequences, 1), t, 1 << 40}:
                    assert [size(t, sequences, heads_q, heads, D, most_new, n) for n in longest] == row
            before = row
        assert before[-1] <= 1 << 28


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,heads,D", [(8, 2, 64), (32, 1, 128), (4, 4, 256)])
def test_one_for_all_calls(seed, H, heads, D, dtype):
    """Calls of fewer tokens of more or fewer sequences with one buffer: what they give with one of their own."""
    from attention_testlib import Paged, attention, heads_of
    from int8_testlib import assert_near
    import paper_1609_07061_amd as q

    ws = torch.empty(q.qnn_cache_attention_workspace_bytes(600, 1, H, heads, D, 600, 3000), dtype=torch.uint8, device="cuda")
    for lengths, fresh in (([3000], [600]), ([3000], [1]), ([3000, 40], [30, 1]), ([1500] * 20, [1] * 20), ([900] * 60, [10] * 60), ([3000], [200]), ([3000, 2000, 1000], [100, 1, 90])):
        p = Paged(seed, lengths, fresh, heads, D, 16)
        x = heads_of(seed, p.tokens, H, D, dtype)
        ws.fill_(255)
        out = q.qnn_cache_attention(x, *p.args, 0.1, most_new=max(fresh), longest=3000, out=torch.empty_like(x), workspace=ws)
        assert torch.equal(out, q.qnn_cache_attention(x, *p.args, 0.1, most_new=max(fresh), longest=3000))
        if len(lengths) < 4 and max(fresh) < 200:
            assert_near(out, *attention(p, x, 0.1)[:2])


@pytest.mark.gpu
@pytest.mark.parametrize("behind", [0, 500, 2500, 9000])
def test_tokens_of_no_sequence(seed, behind):
    """Few tokens of long sequences in a call of many: fewer parts, the same results, and the others left alone."""
    from attention_testlib import Paged, attention, heads_of
    from int8_testlib import assert_near
    import paper_1609_07061_amd as q

    p = Paged(seed, [3000, 700], [1, 2], 2, 64, 16, behind=behind)
    x = heads_of(seed, p.tokens, 32, 64, torch.bfloat16)
    out = torch.full_like(x, 3.0)
    got = q.qnn_cache_attention(x, *p.args, None, most_new=2, longest=3000, out=out)
    want, error, written = attention(p, x, 0.125)
    assert_near(got[written], want[written], error[written])
    assert (out[~written] == 3).all()
