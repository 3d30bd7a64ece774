"""Rows to codes against the definition in 64 bits."""
import math

import pytest
import torch

from int8_testlib import TYPES, U, assert_quantized, generator, normal, placed, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1, 3, 8, 64, 511, 1000, 1025, 2500, 4096, 8200, 33000])
def test_rows(seed, K, dtype):
    import paper_1609_07061_amd as q

    rows = 5 if K > 2048 else 37
    x = normal(generator(seed, rows, K), rows, K).to(dtype)
    x[1] = 0
    codes, scale = q.qnn_rows_quant(x)
    assert_quantized(codes, scale, x.double(), 4 * U)
    for pad, offset in ((1, 1), (5, 3)):
        whole, out = placed(torch.zeros(rows, K, dtype=torch.int8, device="cuda"), pad, offset, 77)
        again = q.qnn_rows_quant(placed(x, pad, offset, float("nan"))[1], out)
        assert torch.equal(again[0], codes) and torch.equal(again[1], scale) and untouched(whole, out, 77)


def test_values(seed):
    import paper_1609_07061_amd as q

    x = normal(generator(seed, 8), 6, 300)
    x[0, 7], x[1, 299], x[2], x[3], x[4] = math.nan, -math.inf, 0.0, x[3] * 1e-41, x[4] * 1e37
    codes, scale = q.qnn_rows_quant(x)
    assert torch.isnan(scale[:2]).all() and (codes[:2] == 0).all() and scale[2] == 0 and (codes[2] == 0).all()
    assert_quantized(codes[4:], scale[4:], x[4:].double(), 4 * U)
    assert q.qnn_rows_quant(x[:0])[0].shape == (0, 300)


def test_beyond_the_caches(seed):
    import paper_1609_07061_amd as q

    x = normal(generator(seed, 9), 20000, 4096).to(torch.bfloat16)
    codes, scale = q.qnn_rows_quant(x)
    some = torch.randint(0, 20000, (300,), generator=generator(seed, 10), device="cuda")
    assert_quantized(codes[some], scale[some], x[some].double(), 4 * U)
    for part in (slice(0, 100), slice(19900, 20000)):
        again = q.qnn_rows_quant(x[part])
        assert torch.equal(again[0], codes[part]) and torch.equal(again[1], scale[part])


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_are_the_definition(seed, dtype):
    """Values of few digits, of which v 127 / max is often the middle between two codes: every code is rint(v 127 / max) in exact arithmetic, ties to even."""
    import paper_1609_07061_amd as q

    g = generator(seed, 11)
    m = torch.randint(-128, 129, (64, 2048), generator=g, device="cuda").double()
    x = (m * 2.0 ** torch.randint(-9, 4, (64, 1), generator=g, device="cuda").double()).to(dtype)
    x[:, 0] = x[:, 0].abs().clamp(min=1)
    y = x.double()
    # in whole numbers: 254 |v| against (2 f + 1) max, in units of the row's power of two
    top = y.abs().amax(dim=1, keepdim=True)
    f = torch.floor(y.abs() * 127 / top)
    f = torch.where((f + 1) * top <= 127 * y.abs(), f + 1, torch.where(f * top > 127 * y.abs(), f - 1, f))
    a, b = 254 * y.abs(), (2 * f + 1) * top
    size = torch.where((a > b) | ((a == b) & (f % 2 == 1)), f + 1, f)
    assert int((a == b).sum()) > 100
    assert torch.equal(q.qnn_rows_quant(x)[0].double(), torch.sign(y) * size)
