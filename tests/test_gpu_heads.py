"""Norm and rotation of heads and their gradient against the formulas in 64 bits."""
import math

import pytest
import torch

from attention_testlib import Rotation, heads_of, norm_rotate, norm_rotate_backward, strided, untouched
from int8_testlib import TYPES, assert_near, generator, normal

pytestmark = pytest.mark.gpu
EPS = 1e-6
# tokens, heads of queries and keys, D, pairs, axes, neighbours
SHAPES = [(1, 1, 1, 16, 8, 1, False), (7, 8, 2, 64, 32, 1, False), (3, 5, 5, 80, 40, 1, True), (33, 4, 1, 128, 64, 3, False), (2, 3, 1, 256, 128, 1, False),
          (20, 32, 8, 128, 64, 3, False), (5, 2, 2, 112, 24, 2, True), (6, 3, 1, 96, 16, 1, False), (4, 2, 1, 240, 0, 1, False), (4099, 2, 1, 64, 32, 1, False),
          (5000, 1, 3, 48, 24, 4, True), (9, 40, 8, 160, 72, 3, False), (1, 0, 4, 32, 16, 1, False)]


def _inputs(seed, shape, dtype, gamma_dtype):
    T, Hq, Hk, D, pairs, axes, neighbours = shape
    g = generator(seed, 77)
    q, k = heads_of(seed, T, Hq, D, dtype), heads_of(seed + 1, T, Hk, D, dtype)
    gammas = [None if gamma_dtype is None or H == 0 else (1 + 0.3 * normal(g, D)).to(gamma_dtype) for H in (Hq, Hk)]
    return q, k, *gammas, Rotation(seed, T, D, pairs, axes, neighbours)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,gamma_dtype", [(t, g) for t in TYPES for g in {t, torch.float32, None}])
def test_forward(seed, shape, dtype, gamma_dtype):
    import paper_1609_07061_amd as q

    x, y, gx, gy, rotation = _inputs(seed, shape, dtype, gamma_dtype)
    got = q.qnn_qk_norm_rotate(x, y, gx, gy, EPS, *rotation.args)
    for out, h, gamma in zip(got, (x, y), (gx, gy)):
        assert_near(out, *norm_rotate(h, gamma, EPS, rotation))
    # strides, addresses, outputs in the inputs' place
    whole_q, sq = strided(x)
    whole_k, sk = strided(y)
    again = q.qnn_qk_norm_rotate(sq, sk, gx, gy, EPS, *rotation.args, q_out=sq, k_out=sk)
    assert again[0] is sq and torch.equal(sq, got[0]) and torch.equal(sk, got[1])
    assert untouched(whole_q, sq, math.nan) and untouched(whole_k, sk, math.nan)
    # heads before tokens
    turned = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (x, y)]
    for a, b in zip(q.qnn_qk_norm_rotate(*turned, gx, gy, EPS, *rotation.args), got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,gamma_dtype", [(t, g) for t in TYPES for g in {t, torch.float32, None}])
def test_backward(seed, shape, dtype, gamma_dtype):
    import paper_1609_07061_amd as q

    x, y, gx, gy, rotation = _inputs(seed, shape, dtype, gamma_dtype)
    da, db = heads_of(seed + 2, *x.shape, dtype, 0.1), heads_of(seed + 3, *y.shape, dtype, 0.1)
    got = q.qnn_qk_norm_rotate_backward(da, db, x, y, gx, gy, EPS, *rotation.args)
    for out, sums, grad, h, gamma in zip(got[:2], got[2:], (da, db), (x, y), (gx, gy)):
        want, error, want_sums, wrong = norm_rotate_backward(grad, h, gamma, EPS, rotation)
        assert_near(out, want, error)
        if gamma is not None:
            assert_near(sums, want_sums, wrong)
    for _ in range(2):  # the same bits again, in the gradients' place
        ca, cb = da.clone(), db.clone()
        again = q.qnn_qk_norm_rotate_backward(ca, cb, x, y, gx, gy, EPS, *rotation.args, out_q=ca, out_k=cb)
        assert all(a is b is None or torch.equal(a, b) for a, b, h in zip(again, got, (x, y, x, y)) if h.shape[1])
    whole, sa = strided(da)
    again = q.qnn_qk_norm_rotate_backward(sa, strided(db)[1], strided(x)[1], strided(y)[1], gx, gy, EPS, *rotation.args, out_q=sa)
    assert torch.equal(sa, got[0]) and torch.equal(again[1], got[1]) and untouched(whole, sa, math.nan)
    if gx is not None and gy is not None:
        assert torch.equal(again[2], got[2]) and torch.equal(again[3], got[3])


@pytest.mark.parametrize("neighbours", [False, True])
def test_backward_is_the_derivative(seed, neighbours):
    """Differences of the formula in 64 bits, at a step that leaves 2^-20 of relative error."""
    import paper_1609_07061_amd as q

    T, H, D = 3, 2, 32
    rotation = Rotation(seed, T, D, 8, 2, neighbours)
    x, grad = heads_of(seed, T, H, D, torch.float32), heads_of(seed + 1, T, H, D, torch.float32)
    gamma = 1 + 0.3 * normal(generator(seed, 5), D)
    value = lambda h, w: (norm_rotate(h, w, EPS, rotation)[0] * grad.double()).sum()
    out, _, sums, _ = q.qnn_qk_norm_rotate_backward(grad, grad, x, x, gamma, gamma, EPS, *rotation.args)
    step = 1e-5
    g = generator(seed, 6)
    for _ in range(8):
        dx, dw = normal(g, T, H, D).double(), normal(g, D).double()
        rate = (value(x.double() + step * dx, gamma.double()) - value(x.double() - step * dx, gamma.double())) / (2 * step)
        assert abs(rate - (out.double() * dx).sum()) <= 1e-5 * (out.double() * dx).abs().sum()
        rate = (value(x.double(), gamma.double() + step * dw) - value(x.double(), gamma.double() - step * dw)) / (2 * step)
        assert abs(rate - (sums.double() * dw).sum()) <= 1e-5 * (sums.double() * dw).abs().sum()


def test_values(seed):
    """Heads that are not finite or zeros stay with themselves; far positions; an axis beyond the axes."""
    import paper_1609_07061_amd as q

    T, H, D = 6, 3, 128
    rotation = Rotation(seed, T, D, axes=2)
    rotation.positions[0] = torch.tensor([2147483647, -2147483648, 1000003, 0, 7, 1 << 20], dtype=torch.int32)
    x = heads_of(seed, T, H, D, torch.float32)
    x[0, 1, 5], x[1, 2, 127], x[2, 0] = math.nan, math.inf, 0.0
    gamma = torch.ones(D, device="cuda")
    out, _ = q.qnn_qk_norm_rotate(x, x[:, :1], gamma, gamma, EPS, *rotation.args)
    fine = torch.ones(T, H, dtype=torch.bool, device="cuda")
    fine[0, 1] = fine[1, 2] = False
    assert not torch.isfinite(out[~fine]).all(dim=1).any() and (out[2, 0] == 0).all()
    want, error = norm_rotate(torch.where(fine[..., None], x, 0.0), gamma, EPS, rotation)
    assert_near(out[fine], want[fine], error[fine])
    beyond = rotation.axis.clone()
    beyond[beyond == 1] = 1 << 30
    beyond[beyond == 0] = -5
    again, _ = q.qnn_qk_norm_rotate(x, x[:, :1], gamma, gamma, EPS, rotation.positions, rotation.freq, beyond)
    assert torch.equal(again[fine], out[fine])


def test_no_tokens(seed):
    import paper_1609_07061_amd as q

    x = torch.zeros(0, 4, 64, device="cuda")
    rotation = Rotation(seed, 0, 64)
    out, _ = q.qnn_qk_norm_rotate(x, x, None, None, EPS, *rotation.args)
    assert out.shape == x.shape
    assert q.qnn_qk_norm_rotate_backward(x, x, x, x, None, None, EPS, *rotation.args)[0].shape == x.shape


def test_captured_gradient(seed):
    """As a graph, replayed on other gradients and with the program's own work between, on a stream of its own."""
    import paper_1609_07061_amd as q

    T, Hq, Hk, D = 700, 4, 2, 64
    rotation = Rotation(seed, T, D)
    x, y, da, db = (heads_of(seed + i, T, H, D, torch.bfloat16) for i, H in enumerate((Hq, Hk, Hq, Hk)))
    gamma = torch.ones(D, device="cuda")
    ws = torch.empty(q.qnn_qk_norm_rotate_backward_workspace_bytes(T, Hq, Hk, D), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(x), torch.empty_like(y), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]
    call = lambda: q.qnn_qk_norm_rotate_backward(da, db, x, y, gamma, gamma, EPS, *rotation.args, *outs, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        da.copy_(heads_of(seed + 10 + i, T, Hq, D, torch.bfloat16))
        want = [t.clone() for t in q.qnn_qk_norm_rotate_backward(da, db, x, y, gamma, gamma, EPS, *rotation.args)]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = q.qnn_qk_norm_rotate_backward(da, db, x, y, gamma, gamma, EPS, *rotation.args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))
