"""Every way that a product of int8 codes can go: sizes that it is chosen for and that it can go wrong at, and that it is the one that runs."""
import pytest
import torch

from int8_testlib import TYPES, generator, placed, untouched
from test_gpu_int8_gemm import _check, _operands

pytestmark = pytest.mark.gpu


def _kernel(call):
    """Name of the one kernel of the library that `call` launches."""
    from torch.profiler import ProfilerActivity, profile

    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    names = [n for e in p.events() for n in ("gemm_stream_kernel", "gemm_panel_kernel", "gemm_tile_kernel") if n in e.name]
    assert len(names) == 1
    return names[0]


# whole 16-byte pieces: streams (16 x 16, 64 x 16, 64 x 32, 64 x 64), panels (64, 128, 256)
PIECES = [("stream", 3, 40, 16), ("stream", 16, 4096, 1040), ("stream", 60, 4000, 4096), ("stream", 120, 4096, 4112), ("stream", 256, 4090, 4096), ("stream", 700, 1000, 4096),
          ("panel", 700, 1000, 272), ("panel", 1200, 1024, 1040), ("panel", 5000, 130, 528), ("panel", 300, 4100, 144), ("panel", 1190, 4000, 1008), ("panel", 5000, 1000, 400),
          ("panel", 130, 20000, 656), ("panel", 5000, 4099, 16), ("panel", 9000, 9001, 256), ("panel", 5003, 4097, 1168), ("panel", 1023, 4090, 2064), ("panel", 4000, 1025, 592), ("panel", 7000, 8000, 128), ("panel", 2560, 16384, 384)]
# any rows: streams, the tiled kernel; fewer codes than a piece
ANY = [("stream", 2, 40, 17), ("stream", 16, 4095, 1001), ("stream", 60, 4000, 4093), ("stream", 120, 4096, 1023), ("stream", 256, 4090, 2047), ("tile", 1999, 1001, 2501), ("tile", 1000, 4001, 17),
       ("tile", 3000, 3000, 127), ("tile", 2500, 2049, 129), ("tile", 4000, 2500, 385), ("tile", 1500, 3000, 250), ("stream", 100, 900, 15), ("stream", 1, 5000, 1), ("stream", 3000, 70, 8)]
# whole 4-byte words: streams, panels (64, 128, 256)
WORDS = [("stream", 150, 1000, 1500), ("stream", 700, 300, 300), ("panel", 300, 4100, 1500), ("panel", 700, 2500, 20), ("panel", 300, 4100, 300), ("panel", 1999, 1001, 2500),
         ("panel", 1500, 3001, 516), ("panel", 4000, 1000, 132), ("panel", 4003, 4097, 1284), ("panel", 9000, 9001, 252), ("panel", 7000, 8000, 124), ("panel", 2500, 2049, 1148)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,M,N,K", PIECES + ANY + WORDS)
def test_way(seed, kind, M, N, K, dtype):
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    for b in (None, bias):
        _check(q.qnn_int8_gemm(A, sA, W, sW, b, dtype=dtype), A, sA, W, sW, b)
    assert _kernel(lambda: q.qnn_int8_gemm(A, sA, W, sW, dtype=dtype)) == f"gemm_{kind}_kernel"


@pytest.mark.parametrize("kind,M,N,K", [("stream", 60, 4000, 4096), ("panel", 1200, 1024, 1040), ("panel", 1190, 4000, 1008), ("panel", 9000, 9001, 256), ("stream", 60, 4000, 4093), ("tile", 1500, 3000, 250),
                                        ("panel", 300, 4100, 308), ("panel", 1500, 3001, 260), ("panel", 9000, 9001, 260)])
def test_way_into_the_middle(seed, kind, M, N, K):
    """Outputs with a pitch, at odd addresses, operands with a pitch: nothing else is written."""
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    pad = 16 if K % 16 == 0 else 4 if kind == "panel" else 5
    a, w = placed(A, pad, pad, 99)[1], placed(W, 2 * pad, 3 * pad, 99)[1]
    for dtype, pad_o, at in ((torch.float32, 3, 1), (torch.bfloat16, 7, 3), (torch.float16, 8, 8)):
        whole, out = placed(torch.zeros(M, N, dtype=dtype, device="cuda"), pad_o, at, 7.0)
        q.qnn_int8_gemm(a, sA, w, sW, bias, out)
        _check(out, A, sA, W, sW, bias)
        assert untouched(whole, out, 7.0)
    assert _kernel(lambda: q.qnn_int8_gemm(a, sA, w, sW, bias, out)) == f"gemm_{kind}_kernel"


def test_beside_each_other(seed):
    """Calls of different ways in flight on two streams."""
    import paper_1609_07061_amd as q

    jobs = [_operands(seed, *s) for s in ((5000, 4096, 512), (16, 4096, 4096), (300, 4100, 160), (1500, 3000, 250))]
    want = [q.qnn_int8_gemm(A, sA, W, sW, b) for A, sA, W, sW, b in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = []
    for _ in range(5):
        for s, (A, sA, W, sW, b) in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(q.qnn_int8_gemm(A, sA, W, sW, b))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % len(jobs)])
