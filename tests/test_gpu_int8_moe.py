"""Mixture-of-experts layer on int8 codes against the definition in 64 bits, and the path through all the calls."""
import math

import pytest
import torch

from int8_testlib import TYPES, U, assert_near, codes_of, generator, moe, normal, placed, silu, untouched

pytestmark = pytest.mark.gpu


def _layer(seed, T, E, H, F):
    g = generator(seed, T, E, H, F)
    scales = lambda *s: 0.5 / math.sqrt(H) / 74 * (normal(g, *s).abs() + 0.5)
    return [codes_of(g, T, H), normal(g, T).abs() / 60 + 0.005, normal(g, T, E), codes_of(g, E, 2 * F, H), scales(E, 2 * F),
            codes_of(g, E, H, F), scales(E, H)]


def _call(q, layer, top, **kw):
    x, sx, logits, w1, s1, w2, s2 = layer
    return q.qnn_int8_moe(x, sx, logits, top, w1, s1, w2, s2, **kw)


def _check(got, layer, top):
    x, sx, logits, w1, s1, w2, s2 = layer
    want, error = moe(x, sx, logits, top, w1, s1, w2, s2)
    gone = torch.isnan(want)
    assert torch.equal(torch.isnan(got), gone)
    assert_near(got[~gone], want[~gone], error[~gone])


SHAPES = [(1, 1, 1, 1, 1), (1, 8, 2, 64, 32), (1, 8, 2, 512, 256), (2, 3, 3, 100, 70), (5, 5, 3, 1000, 700), (16, 16, 4, 256, 128), (17, 4, 1, 300, 200), (20, 8, 2, 512, 300),
          (33, 6, 2, 200, 1500), (64, 8, 8, 130, 65), (64, 2, 1, 128, 2500), (64, 70, 5, 64, 48), (7, 256, 8, 48, 40), (3, 200, 2, 80, 17), (4, 2, 2, 5000, 16), (1, 3, 1, 40, 4200),
          (40, 1, 1, 256, 2049), (64, 5, 4, 96, 1536), (50, 9, 4, 100, 1300), (64, 3, 2, 64, 2048), (10, 4, 3, 96, 624), (64, 6, 6, 48, 10), (30, 4, 1, 80, 6), (9, 12, 4, 2048, 2048), (3, 12, 4, 4096, 1024), (40, 16, 4, 2048, 1536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,top,H,F", SHAPES)
def test_layer(seed, T, E, top, H, F, dtype):
    import paper_1609_07061_amd as q

    layer = _layer(seed, T, E, H, F)
    got = _call(q, layer, top, dtype=dtype)
    assert got.shape == (T, H) and got.dtype == dtype
    _check(got, layer, top)
    assert torch.equal(got, _call(q, layer, top, dtype=dtype))  # the same sums in the same order


@pytest.mark.parametrize("T", [6, 30])
def test_masked_and_tied_logits(seed, T):
    import paper_1609_07061_amd as q

    layer = _layer(seed, T, 7, 96, 80)
    l = layer[2]
    low = torch.finfo(torch.float32).min
    l[0] = -math.inf                          # nobody
    l[1] = -math.inf
    l[1, 4] = 0.5                             # one of three
    l[2] = 1.0                                # the first three
    l[3] = low                                # masked with the lowest value: the first three again
    l[4, 2] = math.nan
    l[5, 3] = math.inf
    if T > 6:
        l[6] = low
        l[6, 6] = 2.0                         # the others have no weight
        l[7] = torch.tensor([0.0, -0.0, 0.0, -0.0, 0.0, -0.0, 0.0])  # no order between the zeros
        l[8] = torch.tensor([-1e30, 3.0, -200.0, 1e-45, 0.0, -1e-45, -math.inf])
        l[9:] = -math.inf
        l[9:, 1] = 0.0                        # all the others on one expert
    got = _call(q, layer, 3, dtype=torch.float32)
    assert (got[0] == 0).all() and torch.isnan(got[4:6]).all()
    _check(got, layer, 3)


@pytest.mark.parametrize("T,E", [(9, 70), (64, 256)])
def test_masked_logits_of_many_experts(seed, T, E):
    import paper_1609_07061_amd as q

    layer = _layer(seed, T, E, 64, 40)
    l = layer[2]
    l[0] = -math.inf
    l[1] = -math.inf
    l[1, E - 1] = 0.5
    l[2] = 1.0                                # the first five
    l[3] = torch.finfo(torch.float32).min
    l[4, 2] = math.nan
    l[5, E - 2] = math.inf
    l[6, : E - 3] = -math.inf                 # three of five
    l[7] = 0.0
    l[7, ::2] = -0.0
    l[8:] = -math.inf
    l[8:, 17:22] = torch.arange(5.0)          # all the others on five experts
    got = _call(q, layer, 5, dtype=torch.float32)
    assert (got[0] == 0).all() and torch.isnan(got[4:6]).all()
    _check(got, layer, 5)


def test_values(seed):
    """Tokens without a value, of zeros, and activations that overflow."""
    import paper_1609_07061_amd as q

    layer = _layer(seed, 5, 4, 64, 48)
    layer[0][0] = 0
    layer[1][1] = math.nan
    layer[1][2] = 1e30      # gate * up beyond fp32
    layer[1][3] = 0.0
    got = _call(q, layer, 2, dtype=torch.float32)
    assert (got[[0, 3]] == 0).all() and torch.isnan(got[1:3]).all()
    layer[1][1:3] = 0.01
    _check(_call(q, layer, 2, dtype=torch.float32)[4:], [t[4:] if i < 3 else t for i, t in enumerate(layer)], 2)


@pytest.mark.parametrize("T,pad,offset", [(3, 1, 1), (3, 16, 16), (20, 5, 3)])
def test_strides(seed, T, pad, offset):
    import paper_1609_07061_amd as q

    layer = _layer(seed, T, 5, 130, 77)
    want = _call(q, layer, 2)
    x, sx, logits, w1, s1, w2, s2 = layer
    there = [placed(x, pad, offset, 55)[1], sx, placed(logits, pad, offset, math.nan)[1], placed(w1.reshape(-1, 130), pad, offset, 55)[1].unflatten(0, (5, 154)), s1,
             placed(w2.reshape(-1, 77), pad + 1, offset, 55)[1].unflatten(0, (5, 130)), s2]
    whole, out = placed(torch.zeros_like(want), pad, offset, 7.0)
    workspace = torch.full((q.qnn_int8_moe_workspace_bytes(T, 2, 77) + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN wherever it is read unwritten)
    assert torch.equal(_call(q, there, 2, out=out, workspace=workspace[:-4096]), want)
    assert untouched(whole, out, 7.0) and (workspace[-4096:] == 0xFF).all()


@pytest.mark.parametrize("T,log_pitch", [(3, 26), (3, 27), (40, 26)])
def test_offsets_beyond_32_bits(seed, T, log_pitch):
    """Experts that lie 4 GiB apart, rows of one that do."""
    import paper_1609_07061_amd as q

    E, H, F, pitch = 3, 48, 16, 1 << log_pitch
    layer = _layer(seed, T, E, H, F)
    want = _call(q, layer, 2, dtype=torch.float32)
    far = list(layer)
    for i in (3, 5):
        w = layer[i]
        far[i] = torch.empty((E * w.shape[1] - 1) * pitch + w.shape[2], dtype=torch.int8, device="cuda").as_strided(w.shape, (w.shape[1] * pitch, pitch, 1))
        far[i].copy_(w)
    assert torch.equal(_call(q, far, 2, dtype=torch.float32), want)
    _check(want, layer, 2)


def test_graph(seed):
    import paper_1609_07061_amd as q

    layer = _layer(seed, 4, 6, 128, 96)
    out, ws = torch.zeros(4, 128, device="cuda"), torch.zeros(q.qnn_int8_moe_workspace_bytes(4, 2, 96), dtype=torch.uint8, device="cuda")
    _call(q, layer, 2, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _call(q, layer, 2, out=out, workspace=ws)
    for i in range(4):
        layer[0].copy_(codes_of(generator(seed, i), 4, 128))
        layer[2].copy_(normal(generator(seed, 10 + i), 4, 6))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _call(q, layer, 2, dtype=torch.float32))


def test_feed_forward_path(seed):
    """Norm, product, gated activation, product: every step against the step's definition on the codes that it was given."""
    import paper_1609_07061_amd as q

    T, H, F = 50, 320, 448
    g = generator(seed, 5)
    x, res, gamma = normal(g, T, H).bfloat16(), normal(g, T, H).bfloat16(), torch.ones(H, device="cuda").bfloat16()
    w1, w2 = codes_of(g, 2 * F, H), codes_of(g, H, F)
    s1, s2 = torch.full((2 * F,), 0.001, device="cuda"), torch.full((H,), 0.001, device="cuda")
    codes, scale, h = q.qnn_rms_norm_quant(x, gamma, 1e-5, res)
    u = q.qnn_int8_gemm(codes, scale, w1, s1)
    a, sa = q.qnn_silu_gate_quant(u[:, :F], u[:, F:])
    y = q.qnn_int8_gemm(a, sa, w2, s2)
    v = (codes.double() * scale.double()[:, None]) @ (w1.double() * 0.001).t()
    assert ((u.double() - v).abs() <= 2.0 ** -8 * v.abs() + 1e-30).all()
    z = silu(u[:, :F].double()) * u[:, F:].double()
    assert ((a.double() * sa.double()[:, None] - z).abs() <= 0.5001 * z.abs().amax(dim=1, keepdim=True) / 127).all()
    v = (a.double() * sa.double()[:, None]) @ (w2.double() * 0.001).t()
    assert ((y.double() - v).abs() <= 2.0 ** -8 * v.abs() + 1e-30).all()
