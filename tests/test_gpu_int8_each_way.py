"""Every way that a product of int8 codes can go, told by the kernel's own template arguments: each at its shortest rows, at ragged edges, in the middle of
larger matrices and next to other ways."""
import pytest
import torch

from int8_testlib import TYPES, placed, untouched
from test_gpu_int8_gemm import _check, _operands

pytestmark = pytest.mark.gpu

# columns / 16, rows / 16, waves, stages, layout (0: whole pieces, 2: any rows, 3: fewer codes than a piece)
STREAM = "gemm_stream_kernel<float,{},(qnn::int8::Layout){}>"
# waves down and across, rows and columns a wave / 32, groups in LDS, workgroups on a compute unit, words
PANEL = "gemm_panel_kernel<float,qnn::int8::panel::Shape<{}>>"
WAYS = {
    "pieces 16 x 16": STREAM.format("1,1,8,2", 0), "pieces 64 x 16": STREAM.format("1,4,8,2", 0),
    "pieces 64 x 32": STREAM.format("2,4,8,1", 0), "pieces 64 x 64": STREAM.format("4,4,8,1", 0),
    "any 16 x 16": STREAM.format("1,1,8,2", 2), "any 64 x 16": STREAM.format("1,4,8,1", 2),
    "any 64 x 32": STREAM.format("2,4,8,1", 2), "any 64 x 64": STREAM.format("4,4,8,1", 2),
    "any 128 x 128": "gemm_tile_kernel<float>", "short": STREAM.format("1,1,8,1", 3),
    "panel 64": PANEL.format("2,2,1,1,4,2,false"), "panel 128, eight waves": PANEL.format("2,4,2,1,4,1,false"),
    "panel 128": PANEL.format("2,2,2,2,2,2,false"), "panel 256": PANEL.format("2,4,4,2,2,1,false"),
    "words 64": PANEL.format("2,2,1,1,4,2,true"), "words 128": PANEL.format("2,2,2,2,2,2,true"), "words 256": PANEL.format("2,4,4,2,2,1,true"),
}

# Sizes at which the rule (for 256 compute units) takes each way: the first for operands and outputs with a pitch too
SIZES = [
    ("pieces 16 x 16", 63, 65, 16), ("pieces 16 x 16", 3, 1001, 4112), ("pieces 64 x 16", 129, 500, 16), ("pieces 64 x 16", 63, 2049, 16), ("pieces 64 x 16", 60, 4000, 4096),
    ("pieces 64 x 32", 257, 1001, 16), ("pieces 64 x 32", 120, 4096, 4112), ("pieces 64 x 64", 256, 4090, 4096), ("pieces 64 x 64", 190, 3901, 4112),
    ("any 16 x 16", 63, 65, 21), ("any 16 x 16", 16, 4095, 1001), ("any 64 x 16", 257, 500, 21), ("any 64 x 16", 60, 4000, 4093), ("any 64 x 32", 257, 1001, 21),
    ("any 64 x 32", 120, 4096, 1023), ("any 64 x 64", 129, 3001, 261), ("any 64 x 64", 256, 4090, 2047),
    ("any 128 x 128", 1500, 3000, 250), ("any 128 x 128", 6000, 130, 21), ("any 128 x 128", 129, 8001, 21), ("any 128 x 128", 2500, 2049, 129), ("any 128 x 128", 1999, 1001, 2501),
    ("short", 100, 900, 15), ("short", 1, 5000, 1),
    ("panel 64", 129, 3001, 16), ("panel 64", 700, 1000, 272), ("panel 64", 5000, 130, 528), ("panel 64", 1200, 1024, 1040),
    ("panel 128, eight waves", 1500, 2049, 400), ("panel 128, eight waves", 500, 8001, 400), ("panel 128, eight waves", 500, 4097, 1024), ("panel 128, eight waves", 1023, 4090, 2064),
    ("panel 128", 1500, 4097, 144), ("panel 128", 1000, 8001, 128), ("panel 128", 4000, 1025, 592), ("panel 128", 1190, 4000, 1008),
    ("panel 256", 3000, 5000, 128), ("panel 256", 2000, 8001, 128), ("panel 256", 2000, 4097, 400), ("panel 256", 5003, 4097, 1168), ("panel 256", 9000, 9001, 256), ("panel 256", 5000, 4099, 16),
    ("words 64", 129, 3001, 516), ("words 64", 6000, 130, 20), ("words 64", 129, 8001, 20), ("words 64", 300, 4100, 1500),
    ("words 128", 500, 4097, 20), ("words 128", 257, 8001, 20), ("words 128", 1500, 3001, 516), ("words 128", 2500, 2049, 1148),
    ("words 256", 2000, 4097, 132), ("words 256", 3000, 4097, 20), ("words 256", 2000, 8001, 20), ("words 256", 4003, 4001, 1284), ("words 256", 4000, 4000, 4004),
]
FIRST = [next(s for s in SIZES if s[0] == way) for way in WAYS]


def _way(call):
    """The way of the one product that `call` (with float32 outputs) launches."""
    from torch.profiler import ProfilerActivity, profile

    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    names = [e.name.replace(" ", "") for e in p.events() if "gemm_" in e.name]
    assert len(names) == 1
    way = [w for w, kernel in WAYS.items() if kernel in names[0]]
    assert len(way) == 1, names
    return way[0]


def test_every_way_is_listed():
    assert all(any(s[0] == way for s in SIZES) for way in WAYS)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("way,M,N,K", SIZES)
def test_dense(seed, way, M, N, K, dtype):
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    for b in (None, bias):
        _check(q.qnn_int8_gemm(A, sA, W, sW, b, dtype=dtype), A, sA, W, sW, b)
    if dtype == torch.float32:
        assert _way(lambda: q.qnn_int8_gemm(A, sA, W, sW, dtype=dtype)) == way


@pytest.mark.parametrize("way,M,N,K", FIRST)
def test_into_the_middle(seed, way, M, N, K):
    """Outputs with a pitch, at odd addresses, operands with a pitch and other codes around them: nothing else is written."""
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    pad = 16 if K % 16 == 0 else 4 if K % 4 == 0 else 5
    a, w = placed(A, pad, pad, 99)[1], placed(W, 2 * pad, 3 * pad, 99)[1]
    for dtype, pad_o, at in ((torch.bfloat16, 7, 3), (torch.float16, 8, 8), (torch.float32, 3, 1)):
        whole, out = placed(torch.zeros(M, N, dtype=dtype, device="cuda"), pad_o, at, 7.0)
        q.qnn_int8_gemm(a, sA, w, sW, bias, out)
        _check(out, A, sA, W, sW, bias)
        assert untouched(whole, out, 7.0)
    assert _way(lambda: q.qnn_int8_gemm(a, sA, w, sW, bias, out)) == way


def test_beside_each_other(seed):
    """The first size of every way, in flight on a stream of its own."""
    import paper_1609_07061_amd as q

    jobs = [_operands(seed, *s[1:]) for s in FIRST]
    want = [q.qnn_int8_gemm(A, sA, W, sW, b) for A, sA, W, sW, b in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = []
    for _ in range(3):
        for s, (A, sA, W, sW, b) in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(q.qnn_int8_gemm(A, sA, W, sW, b))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % len(jobs)])
