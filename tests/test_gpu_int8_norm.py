"""Root-mean-square norm to codes and its gradient against the formulas in 64 bits, at the widths, types, strides and values where they can go wrong."""
import pytest
import torch

from int8_testlib import HALF, TYPES, U, assert_near, assert_quantized, generator, normal, placed, sum_error, untouched

pytestmark = pytest.mark.gpu
EPS = 1e-5
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 512, 513, 1000, 1024, 1025, 2048, 2500, 4096, 4097, 8192, 8193, 20001]
BACKWARD_WIDTHS = [k for k in WIDTHS if k <= 16384] + [16384]


def _norm(h, gamma, eps=EPS):
    return h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps) * gamma


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", WIDTHS + [32768, 32769, 70001])
def test_norm(seed, K, dtype):
    import paper_1609_07061_amd as q

    g = generator(seed, K)
    rows = 5 if K > 2048 else 37
    x, res, gamma = normal(g, rows, K).to(dtype), (normal(g, rows, K) * 3).to(dtype), (1 + normal(g, K) / 4).to(dtype)
    x[1], res[1] = 0, 0
    x[2] = -res[2]
    for gm in (gamma, gamma.float() * 1.001):
        for residual in (res, None):
            h = x.double() if residual is None else x.double() + res.double()
            codes, scale, total = q.qnn_rms_norm_quant(x, gm, EPS, residual)
            # (sum of squares halved by the root; h, the root, three products and the division by 127)
            assert_quantized(codes, scale, _norm(h, gm.double()), (sum_error(K) / 2 + 8) * U)
            if residual is None:
                assert total is x
            else:
                assert ((total.double() - h).abs() <= (HALF[dtype] + U) * h.abs() + 2.0 ** -25).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,pad,offset", [(64, 0, 1), (100, 3, 1), (1000, 8, 0), (1001, 0, 0), (2500, 1, 5), (4096, 16, 8), (4096, 1, 3), (40001, 3, 1)])
def test_norm_strides(seed, K, pad, offset, dtype):
    import paper_1609_07061_amd as q

    g, rows = generator(seed, K, pad), 9
    x, res, gamma = normal(g, rows, K).to(dtype), normal(g, rows, K).to(dtype), (1 + normal(g, K) / 4).to(dtype)
    want = q.qnn_rms_norm_quant(x, gamma, EPS, res)
    _, xv = placed(x, pad, offset, float("nan"))
    _, rv = placed(res, pad + 2, offset, float("nan"))
    gv = placed(gamma[None], 0, offset, float("nan"))[1][0]
    whole_c, cv = placed(torch.zeros(rows, K, dtype=torch.int8, device="cuda"), pad, offset, 77)
    whole_t, tv = placed(x, pad + 1, offset, 7.0)
    codes, scale, total = q.qnn_rms_norm_quant(xv, gv, EPS, rv, cv, None, tv)
    assert torch.equal(codes, want[0]) and torch.equal(scale, want[1]) and torch.equal(total, want[2])
    assert untouched(whole_c, cv, 77) and untouched(whole_t, tv, 7.0)
    # the sum in the place of an operand
    for which in (0, 1):
        xi, ri = xv.clone(), rv.clone()
        out = q.qnn_rms_norm_quant(xi, gv, EPS, ri, total=(xi, ri)[which])
        assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2]) and out[2] is (xi, ri)[which]


@pytest.mark.parametrize("K", [10, 700, 3000, 33000])
def test_norm_values(seed, K):
    """Rows of zeros, of the smallest and largest numbers, with NaN and infinities."""
    import paper_1609_07061_amd as q

    x = normal(generator(seed, K), 10, K)
    x[0] = 0
    x[1, K // 2] = float("nan")
    x[2, K - 1] = float("inf")
    x[3, 0] = float("-inf")
    x[4] *= 1e-30
    x[5] = 0
    x[5, K - 1] = 1e-42
    x[6] *= 1e15
    x[7] = 3e38
    gamma = torch.ones(K, device="cuda")
    codes, scale, _ = q.qnn_rms_norm_quant(x, gamma, EPS)
    assert torch.isnan(scale[[1, 2, 3, 7]]).all() and (codes[[0, 1, 2, 3, 7]] == 0).all() and scale[0] == 0
    fine = [4, 6, 8, 9]
    assert_quantized(codes[fine], scale[fine], _norm(x[fine].double(), 1.0), (sum_error(K) / 2 + 8) * U)
    assert codes[5, K - 1] == 127 and (codes[5, :K - 1] == 0).all()
    # without eps, and a gamma that leaves nothing
    codes, scale, _ = q.qnn_rms_norm_quant(x, gamma, 0.0)
    assert scale[0] == 0 and (codes[0] == 0).all()
    assert_quantized(codes[8:], scale[8:], _norm(x[8:].double(), 1.0, 0.0), (sum_error(K) / 2 + 8) * U)
    codes, scale, _ = q.qnn_rms_norm_quant(x[8:], torch.zeros(K, device="cuda"), EPS)
    assert (scale == 0).all() and (codes == 0).all()


def _backward(g, h, gamma, z):
    r = 1 / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    wg = g * gamma
    gh = r * (wg - h * r.square() * (wg * h).mean(dim=1, keepdim=True))
    size = r * (wg.abs() + h.abs() * r.square() * (wg * h).abs().mean(dim=1, keepdim=True))  # what the errors are relative to
    return (gh if z is None else gh + z), (g * h * r).sum(dim=0), size + (0 if z is None else z.abs()), (g * h * r).abs().sum(dim=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", BACKWARD_WIDTHS)
def test_backward(seed, K, dtype):
    import paper_1609_07061_amd as q

    g, rows = generator(seed, K, 1), 3 if K > 4096 else 61
    grad, h, z = (normal(g, rows, K).to(dtype) for _ in range(3))
    h[1] = 0
    for gamma in ((1 + normal(g, K) / 4).to(dtype), 1 + normal(g, K) / 4):
        for extra in (z, None):
            gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, EPS, extra)
            want = _backward(grad.double(), h.double(), gamma.double(), None if extra is None else z.double())
            assert_near(gh, want[0], (2 * sum_error(K) + 10) * U * want[2])
            assert_near(gw, want[1], (sum_error(K) / 2 + rows + 10) * U * want[3])


@pytest.mark.parametrize("rows,K", [(1, 64), (513, 64), (4099, 200), (2049, 1024), (1500, 2500), (3000, 129)])
def test_backward_many_rows(seed, rows, K):
    import paper_1609_07061_amd as q

    g = generator(seed, rows, K)
    grad, h, gamma = normal(g, rows, K), normal(g, rows, K), 1 + normal(g, K) / 4
    gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, EPS)
    want = _backward(grad.double(), h.double(), gamma.double(), None)
    assert_near(gh, want[0], (2 * sum_error(K) + 10) * U * want[2])
    # (up to 512 partial sums of rows / 512 rows)
    assert_near(gw, want[1], (sum_error(K) / 2 + rows / 512 + 4 + 16 + 10 + 10) * U * want[3])
    again = q.qnn_rms_norm_backward(grad, h, gamma, EPS)
    assert torch.equal(gh, again[0]) and torch.equal(gw, again[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,pad,offset", [(100, 3, 1), (1001, 0, 0), (2500, 1, 5), (4096, 1, 3)])
def test_backward_strides(seed, K, pad, offset, dtype):
    import paper_1609_07061_amd as q

    g, rows = generator(seed, K, pad, 2), 11
    grad, h, z, gamma = normal(g, rows, K).to(dtype), normal(g, rows, K).to(dtype), normal(g, rows, K).to(dtype), (1 + normal(g, K) / 4).to(dtype)
    want = q.qnn_rms_norm_backward(grad, h, gamma, EPS, z)
    views = [placed(t, pad + i, offset, float("nan"))[1] for i, t in enumerate((grad, h, z))]
    whole, out = placed(z, pad, offset + 1, 7.0)
    got = q.qnn_rms_norm_backward(views[0], views[1], placed(gamma[None], 0, offset, float("nan"))[1][0], EPS, views[2], out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and untouched(whole, out, 7.0)
    got = q.qnn_rms_norm_backward(views[0], views[1], gamma, EPS, views[2], views[2])  # the gradient in the place of the one it is added to
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("K", [5, 600, 2500])
def test_backward_against_differences(seed, K):
    """The derivative of sum(grad * y) along a direction in h and in gamma, by central differences in 64 bits."""
    import paper_1609_07061_amd as q

    g, rows = generator(seed, K, 3), 7
    grad, h, gamma, dh, dg = normal(g, rows, K), normal(g, rows, K), 1 + normal(g, K) / 4, normal(g, rows, K), normal(g, K)
    gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, EPS)

    def value(step):
        return (grad.double() * _norm(h.double() + step * dh.double(), gamma.double() + step * dg.double())).sum()

    step = 1e-5
    slope = (value(step) - value(-step)) / (2 * step)
    got = (gh.double() * dh.double()).sum() + (gw.double() * dg.double()).sum()
    # differences: step^2 times third derivatives, and 2^-52 / step; kernel: fp32
    size = _backward(grad.double(), h.double(), gamma.double(), None)
    bound = (2 * sum_error(K) + 10) * U * ((size[2] * dh.double().abs()).sum() + (size[3] * dg.double().abs()).sum())
    assert (got - slope).abs() <= bound + 1e-6 * (1 + slope.abs()) + 1e-8 * rows * K


def _far_apart(t, pitch):
    """The rows of t, `pitch` elements apart."""
    whole = torch.empty((t.shape[0] - 1) * pitch + t.shape[1], dtype=t.dtype, device="cuda")
    view = whole.as_strided(t.shape, (pitch, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("K", [256, 333])
def test_offsets_beyond_32_bits(seed, K):
    """Rows that lie more than 4 GiB apart."""
    import paper_1609_07061_amd as q

    g, pitch = generator(seed, K, 9), (1 << 31) + 72
    x, res, grad, gamma = normal(g, 3, K).bfloat16(), normal(g, 3, K).bfloat16(), normal(g, 3, K).bfloat16(), (1 + normal(g, K) / 4).bfloat16()
    want, want_grad = q.qnn_rms_norm_quant(x, gamma, EPS, res), q.qnn_rms_norm_backward(grad, x, gamma, EPS, res)
    far = _far_apart(x, pitch)
    got = q.qnn_rms_norm_backward(grad, far, gamma, EPS, res)
    assert torch.equal(got[0], want_grad[0]) and torch.equal(got[1], want_grad[1])
    codes = _far_apart(torch.zeros(3, K, dtype=torch.int8, device="cuda"), pitch)
    got = q.qnn_rms_norm_quant(far, gamma, EPS, res, codes, None, far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    got = q.qnn_rms_norm_backward(grad, x, gamma, EPS, res, far)
    assert torch.equal(got[0], want_grad[0])
