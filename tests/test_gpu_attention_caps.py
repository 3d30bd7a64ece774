"""Capped scores against the definition in 64 bits, from caps that hold everything to caps that nothing reaches, in all types and on both kernels."""
import pytest
import torch

from attention_testlib import Paged, attention, heads_of
from int8_testlib import U, assert_near

pytestmark = pytest.mark.gpu
NAMES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CAPS = [1e-30, 0.5, 7.0, 50.0, 64.0, 65.0, 1e3, 1e4, 1e5, 1e8, 1e20, 1e35, 1.5e38, 3e38]


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh,heads,D", [(1, 2, 128), (40, 2, 64), (400, 2, 64), (220, 1, 256)])  # few rows, more, and those of the kernel for many
@pytest.mark.parametrize("bias", [False, True])
def test_caps(seed, fresh, heads, D, bias, type):
    import paper_1609_07061_amd as q

    H = 4 * heads
    p = Paged(seed, [500, 60], [fresh, 1], heads, D, 16)
    slopes = 2.0 ** -torch.arange(1, H + 1, device="cuda", dtype=torch.float32) if bias else None
    for factor in (0.1, 3.0):
        x = heads_of(seed, p.tokens, H, D, NAMES[type], factor)
        largest = 127 * p.cache[3].max().double()
        for cap in CAPS:
            want, error, written = attention(p, x, D ** -0.5, cap, slopes)
            if type != "f32" and cap <= 64:
                # size - 2 size / (1 + 2^y): the exponent, the sum and the quotient are each off by U or 2 U of a factor up to 1, the product with 2 size doubles that, and the last
                # difference is rounded: 8 U of the cap, for the weight and for the sum
                error = error + 2 * 8 * U * cap * largest
            assert_near(q.qnn_cache_attention(x, *p.args, None, cap, slopes, most_new=fresh, longest=500)[written], want[written], error[written])


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh", [1, 400])
def test_a_cap_that_nothing_reaches(seed, fresh, type):
    """The same as without one, within what either is off by."""
    import paper_1609_07061_amd as q

    p = Paged(seed, [900], [fresh], 1, 64, 16)
    x = heads_of(seed, fresh, 4, 64, NAMES[type], 2.0)
    plain, error, _ = attention(p, x, 0.125)
    for cap in (1e12, 1e30, 3e38):
        assert_near(q.qnn_cache_attention(x, *p.args, 0.125, cap, most_new=fresh, longest=900), plain, error)
