"""The norm and its gradient on rows whose values or sums are hard to hold: what the forward call counts as not finite has no gradient either."""
import math

import pytest
import torch

from int8_testlib import U, assert_near, assert_quantized, generator, normal, sum_error

pytestmark = pytest.mark.gpu
EPS = 1e-5
# a width for each number of lanes and of values a lane
BACKWARD_WIDTHS = [5, 300, 1000, 1500, 2500, 4097, 16384]


def backward(g, h, gamma, eps):
    """(gradient at h, rows' parts of the gradient at gamma, what the errors of the first are relative to), in 64 bits"""
    r = 1 / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps)
    wg, unit = g * gamma, h * r
    size = r * (wg.abs() + unit.abs() * (wg * unit).abs().mean(dim=1, keepdim=True))
    return r * (wg - unit * (wg * unit).mean(dim=1, keepdim=True)), g * unit, size


def check_backward(got, g, h, gamma, eps, factor):
    """`factor`: of U, for the two sums of a row."""
    want = backward(g.double(), h.double(), gamma.double(), eps)
    assert_near(got[0], want[0], (2 * factor + 10) * U * want[2])
    assert_near(got[1], want[1].sum(dim=0), (factor / 2 + len(h) + 10) * U * want[1].abs().sum(dim=0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", BACKWARD_WIDTHS)
def test_rows_that_are_not_finite(seed, K, dtype):
    import paper_1609_07061_amd as q

    g = generator(seed, K, 4)
    h, grad, z, gamma = normal(g, 9, K).to(dtype), normal(g, 9, K).to(dtype), normal(g, 9, K).to(dtype), (1 + normal(g, K) / 4).to(dtype)
    h[0, K // 2] = math.nan
    h[1, K - 1] = math.inf
    h[2, 0] = -math.inf
    h[3] = 3e38                       # a mean square beyond fp32
    h[4] = 2e19
    h[4, 1::2] = -2e19
    h[5] = 0
    h[6] *= 1e-30
    bad, fine = [0, 1, 2, 3, 4], [5, 6, 7, 8]
    assert torch.equal(torch.isnan(q.qnn_rms_norm_quant(h, gamma, EPS)[1]).cpu(), torch.tensor([i in bad for i in range(9)]))
    for extra in (None, z):
        gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, EPS, extra)
        assert torch.isnan(gh[bad]).all() and torch.isnan(gw).all()
        rest = q.qnn_rms_norm_backward(grad[fine], h[fine], gamma, EPS, None if extra is None else extra[fine])
        assert torch.equal(gh[fine], rest[0]) and torch.isfinite(rest[0]).all() and torch.isfinite(rest[1]).all()
        # each row by itself
        for i in bad:
            one = q.qnn_rms_norm_backward(grad[i : i + 1], h[i : i + 1], gamma, EPS, None if extra is None else extra[i : i + 1])
            assert torch.isnan(one[0]).all() and torch.isnan(one[1]).all()
    check_backward(q.qnn_rms_norm_backward(grad[fine], h[fine], gamma, EPS), grad[fine], h[fine], gamma, EPS, sum_error(K))


@pytest.mark.parametrize("K", BACKWARD_WIDTHS)
def test_gradient_that_is_not_finite(seed, K):
    """A value of the incoming gradient that is not finite shows in its row and in its own column of the weight's gradient, nowhere else."""
    import paper_1609_07061_amd as q

    g = generator(seed, K, 5)
    h, grad, gamma = normal(g, 4, K), normal(g, 4, K), 1 + normal(g, K) / 4
    want = q.qnn_rms_norm_backward(grad, h, gamma, EPS)
    for value in (math.nan, math.inf):
        bad = grad.clone()
        bad[2, K - 2] = value
        gh, gw = q.qnn_rms_norm_backward(bad, h, gamma, EPS)
        rows, columns = [0, 1, 3], [k for k in range(K) if k != K - 2]
        assert torch.equal(gh[rows], want[0][rows]) and torch.equal(gw[columns], want[1][columns])
        assert not torch.isfinite(gh[2]).any() and not torch.isfinite(gw[K - 2])


@pytest.mark.parametrize("K", [10, 700, 3000, 33000])
def test_squares_out_of_range(seed, K):
    """Rows whose squares fp32 does not hold: exact or marked, never an approximation."""
    import paper_1609_07061_amd as q

    x, gamma = normal(generator(seed, K, 6), 10, K), torch.ones(K, device="cuda")
    sizes = [1e-18, 1e-21, 1e-23, 1e-25, 1e-30, 1e-40, 0.0, 1e17, 3e19, 1.0]
    x *= torch.tensor(sizes, device="cuda")[:, None]
    x[9] = 0
    x[9, K // 2] = 1e-22  # one value only
    codes, scale, _ = q.qnn_rms_norm_quant(x, gamma, 0.0)
    marked = [1, 2, 3, 4, 5, 8, 9]
    assert torch.isnan(scale[marked]).all() and (codes[marked] == 0).all()
    assert scale[6] == 0 and (codes[6] == 0).all()
    y = x.double() / torch.sqrt(x.double().square().mean(dim=1, keepdim=True))
    assert_quantized(codes[[0, 7]], scale[[0, 7]], y[[0, 7]], (sum_error(K) / 2 + 9) * U)  # (a square's rounding is up to 2 U at 2^-126)
    # nothing left of any of them, whatever the sum is
    codes, scale, _ = q.qnn_rms_norm_quant(x[[1, 4, 5, 6]], 0 * gamma, 0.0)
    assert (scale == 0).all() and (codes == 0).all()
    # a mean square and an eps that fp32 holds one by one
    big = torch.zeros(1, K, device="cuda")
    big[0, 0] = 1.8e19
    assert torch.isfinite(q.qnn_rms_norm_quant(big, gamma, 1e-5)[1]).all()
    assert torch.isnan(q.qnn_rms_norm_quant(big[:, :1], gamma[:1], 3e38)[1]).all()


@pytest.mark.parametrize("K", BACKWARD_WIDTHS)
def test_gradient_of_squares_out_of_range(seed, K):
    import paper_1609_07061_amd as q

    g = generator(seed, K, 7)
    h, grad, gamma = normal(g, 7, K), normal(g, 7, K), 1 + normal(g, K) / 4
    h *= torch.tensor([1e-18, 1e-21, 1e-25, 1e-40, 0.0, 1e17, 1.0], device="cuda")[:, None]
    fine = [0, 5, 6]
    gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, 0.0)
    assert not torch.isfinite(gh[1:5]).any() and not torch.isfinite(gw).any()
    rest = q.qnn_rms_norm_backward(grad[fine], h[fine], gamma, 0.0)
    assert torch.equal(rest[0], gh[fine])
    check_backward(rest, grad[fine], h[fine], gamma, 0.0, sum_error(K) + 2)
