"""Norm, gated activation and their gradients on matrices beyond 128 MB, which pass the caches: against the same rows in smaller calls, bit for bit, and against
the formulas in 64 bits."""
import pytest
import torch

from int8_testlib import TYPES, U, assert_near, assert_quantized, generator, normal, placed, silu, sum_error, untouched

pytestmark = pytest.mark.gpu
EPS = 1e-5
LIMIT = 128e6  # bytes of a call's matrices
# fewer values than a lane takes, a wave, four and sixteen waves a row, rows that are read twice
WIDTHS = [5, 9, 1001, 2501, 4097, 9001, 33001]
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
@pytest.mark.parametrize("K", WIDTHS)
def test_norm(seed, K, dtype):
    import paper_1609_07061_amd as q

    w = dtype.itemsize
    rows = _rows(K, 3 * w + 1)
    g = generator(seed, K, 11)
    x, res, gamma = normal(g, rows, K).to(dtype), (normal(g, rows, K) * 3).to(dtype), (1 + normal(g, K) / 4).to(dtype)
    call = lambda x, res: q.qnn_rms_norm_quant(x, gamma, EPS, res)
    want = _in_parts(call, rows, x, res)
    got = call(x, res)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    h = x.double() + res.double()
    assert_quantized(want[0], want[1], h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS) * gamma.double(), (sum_error(K) / 2 + 8) * U)
    del h
    if dtype == torch.float32:
        assert ["NormSource<float,true>" in n for n in _kernel(lambda: call(x, res), "quant_rows")] == [True]
    for pad, offset in LAYOUTS:
        xv, rv = placed(x, pad, offset, float("nan"))[1], placed(res, pad + 1, offset, float("nan"))[1]
        whole_c, cv = placed(torch.zeros(rows, K, dtype=torch.int8, device="cuda"), pad, offset, 77)
        whole_t, tv = placed(x, pad + 2, offset, 7.0)
        codes, scale, total = q.qnn_rms_norm_quant(xv, gamma, EPS, rv, cv, None, tv)
        assert torch.equal(codes, want[0]) and torch.equal(scale, want[1]) and torch.equal(total, want[2])
        assert untouched(whole_c, cv, 77) and untouched(whole_t, tv, 7.0)
        del whole_c, whole_t, cv, tv, codes, total
        # the sum in the place of an operand
        out = q.qnn_rms_norm_quant(xv, gamma, EPS, rv, total=rv)
        assert torch.equal(out[0], want[0]) and torch.equal(rv, want[2])
        rv.copy_(res)
        out = q.qnn_rms_norm_quant(xv, gamma, EPS, rv, total=xv)
        assert torch.equal(out[0], want[0]) and torch.equal(xv, want[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [5, 9, 513, 1001, 1025, 2501, 4097, 9001, 16384])
def test_norm_gradient(seed, K, dtype):
    import paper_1609_07061_amd as q

    rows = _rows(K, 3 * dtype.itemsize)
    g = generator(seed, K, 12)
    grad, h, z, gamma = normal(g, rows, K).to(dtype), normal(g, rows, K).to(dtype), normal(g, rows, K).to(dtype), 1 + normal(g, K) / 4
    hd, gd = h.double(), grad.double()
    r = 1 / torch.sqrt(hd.square().mean(dim=1, keepdim=True) + EPS)
    want_w, size_w = (gd * hd * r).sum(dim=0), (gd * hd * r).abs().sum(dim=0)
    wg = gd * gamma.double()
    mean, size = (wg * hd).mean(dim=1, keepdim=True), (wg * hd).abs().mean(dim=1, keepdim=True)
    want, size = r * (wg - hd * r.square() * mean), r * (wg.abs() + hd.abs() * r.square() * size)
    del wg, hd, gd
    for extra in (None, z):
        call = lambda grad, h, z: [q.qnn_rms_norm_backward(grad, h, gamma, EPS, z)[0]]
        small, = _in_parts(call, rows, grad, h, extra)
        gh, gw = q.qnn_rms_norm_backward(grad, h, gamma, EPS, extra)
        assert torch.equal(gh, small)
        more = 0 if extra is None else extra.double()
        assert_near(gh, want + more, (2 * sum_error(K) + 10) * U * (size + abs(more)))
        # (up to 512 partial sums of rows / 512 rows)
        assert_near(gw, want_w, (sum_error(K) / 2 + rows / 512 + 4 + 16 + 10 + 10) * U * size_w)
    if dtype == torch.float32 and K > 8:
        name, = _kernel(lambda: q.qnn_rms_norm_backward(grad, h, gamma, EPS, z), "rms_norm_backward_kernel")
        assert ",true,false>" in name
    del want, size, more
    for pad, offset in LAYOUTS:
        views = [placed(t, pad + i, offset, float("nan"))[1] for i, t in enumerate((grad, h, z))]
        whole, out = placed(z, pad, offset + 1, 7.0)
        got = q.qnn_rms_norm_backward(views[0], views[1], gamma, EPS, views[2], out)
        assert torch.equal(got[0], gh) and torch.equal(got[1], gw) and untouched(whole, out, 7.0)
        q.qnn_rms_norm_backward(views[0], views[1], gamma, EPS, views[2], views[2])
        assert torch.equal(views[2], gh)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F", WIDTHS)
def test_gate(seed, F, dtype):
    import paper_1609_07061_amd as q

    rows = _rows(F, 2 * dtype.itemsize + 1)
    u = (normal(generator(seed, F, 13), rows, 2 * F) * 2).to(dtype)
    gate, up = u[:, :F], u[:, F:]
    want = _in_parts(q.qnn_silu_gate_quant, rows, gate, up)
    got = q.qnn_silu_gate_quant(gate, up)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert_quantized(want[0], want[1], silu(gate.double()) * up.double(), 16 * U)
    if dtype == torch.float32:
        assert ["GateSource<float,true>" in n for n in _kernel(lambda: q.qnn_silu_gate_quant(gate, up), "quant_rows")] == [True]
    for pad, offset in LAYOUTS:
        gv, uv = placed(gate, pad, offset, float("nan"))[1], placed(up, pad + 1, offset + 1, float("nan"))[1]
        whole, out = placed(torch.zeros(rows, F, dtype=torch.int8, device="cuda"), pad, offset, 77)
        got = q.qnn_silu_gate_quant(gv, uv, out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and untouched(whole, out, 77)


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
