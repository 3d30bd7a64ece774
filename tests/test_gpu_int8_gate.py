"""Gated activation to codes and its gradient against the formulas in 64 bits."""
import pytest
import torch

from int8_testlib import TYPES, U, assert_near, assert_quantized, generator, normal, placed, silu, untouched

pytestmark = pytest.mark.gpu
WIDTHS = [1, 3, 8, 64, 511, 1000, 1024, 1025, 2500, 4096, 5000, 8200, 33000]


def _inputs(seed, rows, F, dtype):
    g = generator(seed, rows, F)
    return (normal(g, rows, 2 * F) * 2).to(dtype), normal(g, rows, F).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F", WIDTHS)
def test_gate(seed, F, dtype):
    import paper_1609_07061_amd as q

    rows = 5 if F > 2048 else 37
    u, _ = _inputs(seed, rows, F, dtype)
    u[1] = 0
    y = silu(u[:, :F].double()) * u[:, F:].double()
    codes, scale = q.qnn_silu_gate_quant(u[:, :F], u[:, F:])
    # exp within 2 units, sum, quotient, product, quotient by 127
    assert_quantized(codes, scale, y, 16 * U)
    for pad, offset in ((1, 1), (5, 3)):
        gate, up = placed(u[:, :F], pad, offset, float("nan"))[1], placed(u[:, F:], pad + 1, offset + 1, float("nan"))[1]
        whole, out = placed(torch.zeros(rows, F, dtype=torch.int8, device="cuda"), pad, offset, 77)
        got = q.qnn_silu_gate_quant(gate, up, out)
        assert torch.equal(got[0], codes) and torch.equal(got[1], scale) and untouched(whole, out, 77)


def test_gate_values():
    import paper_1609_07061_amd as q

    F = 300
    gate, up = torch.ones(8, F, device="cuda"), torch.ones(8, F, device="cuda")
    gate[0, 7] = float("nan")
    up[1, 299] = float("inf")
    gate[2, 0] = float("inf")
    gate[3] = -200.0           # exp beyond fp32: zeros
    gate[4] = torch.linspace(-80, 80, F)
    gate[5] = -3.0e38
    up[6] = 1e-36
    up[7] = 0
    codes, scale = q.qnn_silu_gate_quant(gate, up)
    assert torch.isnan(scale[:3]).all() and (codes[:3] == 0).all()
    assert (scale[[3, 5, 7]] == 0).all() and (codes[[3, 5, 7]] == 0).all()
    y = silu(gate.double()) * up.double()
    assert_quantized(codes[[4, 6]], scale[[4, 6]], y[[4, 6]], 16 * U)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,F", [(1, 1), (37, 7), (5, 64), (200, 1001), (13, 4096), (2, 33000)])
def test_gate_backward(seed, rows, F, dtype):
    import paper_1609_07061_amd as q

    u, grad = _inputs(seed, rows, F, dtype)
    gate, up, g = u[:, :F].double(), u[:, F:].double(), grad.double()
    s = torch.sigmoid(gate)
    want = g * up * s * (1 + gate * (1 - s)), g * gate * s
    error = 16 * U * (g * up * s).abs() * (1 + gate.abs()), 16 * U * want[1].abs()
    # (products of small factors may fall below fp32's normal numbers)
    tiny = 2.0 ** -140
    got = q.qnn_silu_gate_backward(grad, u[:, :F], u[:, F:])
    assert_near(got[0], want[0], error[0] + tiny)
    assert_near(got[1], want[1], error[1] + tiny)
    whole_a, a = placed(grad, 3, 1, 7.0)
    whole_b, b = placed(grad, 2, 5, 7.0)
    placed_in = [placed(t, 1, 3, float("nan"))[1] for t in (grad, u[:, :F], u[:, F:])]
    q.qnn_silu_gate_backward(*placed_in, a, b)
    assert torch.equal(a, got[0]) and torch.equal(b, got[1]) and untouched(whole_a, a, 7.0) and untouched(whole_b, b, 7.0)
    q.qnn_silu_gate_backward(*placed_in, placed_in[1], placed_in[2])  # in the place of the inputs
    assert torch.equal(placed_in[1], got[0]) and torch.equal(placed_in[2], got[1])


def test_gate_backward_against_differences(seed):
    import paper_1609_07061_amd as q

    rows, F = 9, 77
    u, grad = _inputs(seed, rows, F, torch.float32)
    d = normal(generator(seed, 9), rows, 2 * F).double()
    got = torch.cat(q.qnn_silu_gate_backward(grad, u[:, :F], u[:, F:]), dim=1).double()

    def value(step):
        v = u.double() + step * d
        return (grad.double() * silu(v[:, :F]) * v[:, F:]).sum()

    step = 1e-5
    slope = (value(step) - value(-step)) / (2 * step)
    size = (grad.double().abs() * (u[:, :F].double().abs() + 1) * (u[:, F:].double().abs() + 1)).sum() * d.abs().max()
    assert ((got * d).sum() - slope).abs() <= 16 * U * size + 1e-6 * (1 + slope.abs())


@pytest.mark.parametrize("gate,value", [(-120.0, 0.0), (120.0, 1.0)])
def test_gate_backward_far_out(gate, value):
    """Where the exponential is beyond fp32 or nothing, the derivative is that of 0 or of up * gate."""
    import paper_1609_07061_amd as q

    x, one = torch.full((3, 40), gate, device="cuda"), torch.ones(3, 40, device="cuda")
    a, b = q.qnn_silu_gate_backward(one, x, one)
    assert (a == value).all() and (b == value * gate).all()


def test_offsets_beyond_32_bits(seed):
    """Rows that lie more than 4 GiB apart."""
    import paper_1609_07061_amd as q

    F, pitch = 333, (1 << 31) + 72
    u, grad = _inputs(seed, 3, F, torch.bfloat16)
    want, want_grad = q.qnn_silu_gate_quant(u[:, :F], u[:, F:]), q.qnn_silu_gate_backward(grad, u[:, :F], u[:, F:])
    far = torch.empty(2 * pitch + 2 * F, dtype=torch.bfloat16, device="cuda").as_strided((3, 2 * F), (pitch, 1))
    far.copy_(u)
    got = q.qnn_silu_gate_quant(far[:, :F], far[:, F:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = q.qnn_silu_gate_backward(grad, far[:, :F], far[:, F:], far[:, :F], far[:, F:])
    assert torch.equal(got[0], want_grad[0]) and torch.equal(got[1], want_grad[1])
