"""Gradient of the gated activation on matrices beyond 128 MB, which pass the caches: against the same rows in smaller calls, bit for bit, and against
the formulas in 64 bits."""
import pytest
import torch

from int8_testlib import TYPES, U, assert_near, generator, normal, placed, untouched

pytestmark = pytest.mark.gpu
LIMIT = 128e6  # bytes of a call's matrices
LAYOUTS = [(0, 0), (3, 1), (8, 5)]


def _rows(width, bytes_a_value):
    return int(LIMIT / (width * bytes_a_value)) + 77


def _in_parts(call, rows, *matrices):
    """call(parts of the matrices) for three parts of the rows, each below the limit; the results put together."""
    edges = [0, rows // 3, rows // 2, rows]
    parts = [call(*[None if m is None else m[a:b] for m in matrices]) for a, b in zip(edges, edges[1:])]
    return [torch.cat([p[i] for p in parts]) for i in range(len(parts[0]))]


def _kernel(call, part):
    """Names of the kernels that `call` launches and that have `part` in theirs."""
    from torch.profiler import ProfilerActivity, profile

    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name.replace(" ", "") for e in p.events() if part in e.name]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F", [5, 9, 1001, 2501, 4096])
def test_gate_gradient(seed, F, dtype):
    import paper_1609_07061_amd as q

    rows = _rows(F, 5 * dtype.itemsize)
    g = generator(seed, F, 14)
    u, grad = (normal(g, rows, 2 * F) * 2).to(dtype), normal(g, rows, F).to(dtype)
    want = _in_parts(lambda *m: q.qnn_silu_gate_backward(*m), rows, grad, u[:, :F], u[:, F:])
    got = q.qnn_silu_gate_backward(grad, u[:, :F], u[:, F:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    gate, up, gd = u[:, :F].double(), u[:, F:].double(), grad.double()
    s = torch.sigmoid(gate)
    # (products of small factors may fall below fp32's normal numbers)
    assert_near(want[0], gd * up * s * (1 + gate * (1 - s)), 16 * U * (gd * up * s).abs() * (1 + gate.abs()) + 2.0 ** -140)
    assert_near(want[1], gd * gate * s, 16 * U * (gd * gate * s).abs() + 2.0 ** -140)
    del gate, up, gd, s
    if dtype == torch.float32 and F > 8:
        name, = _kernel(lambda: q.qnn_silu_gate_backward(grad, u[:, :F], u[:, F:]), "silu_gate_backward_kernel")
        assert "<float,true,false>" in name
    for pad, offset in LAYOUTS:
        views = [placed(t, pad + i, offset, float("nan"))[1] for i, t in enumerate((grad, u[:, :F], u[:, F:]))]
        whole_a, a = placed(grad, pad, offset + 1, 7.0)
        whole_b, b = placed(grad, pad + 2, offset, 7.0)
        q.qnn_silu_gate_backward(*views, a, b)
        assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and untouched(whole_a, a, 7.0) and untouched(whole_b, b, 7.0)
        q.qnn_silu_gate_backward(*views, views[1], views[2])  # in the place of the inputs
        assert torch.equal(views[1], want[0]) and torch.equal(views[2], want[1])
