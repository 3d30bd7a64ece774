"""Product of int8 codes with scales against the exact sums."""
import pytest
import torch

from int8_testlib import TYPES, U, assert_near, codes_of, generator, normal, placed, untouched

pytestmark = pytest.mark.gpu


def _operands(seed, M, N, K):
    g = generator(seed, M, N, K)
    return codes_of(g, M, K), normal(g, M).abs() + 0.01, codes_of(g, N, K), normal(g, N) * 0.01, normal(g, N)


def _check(got, A, sA, W, sW, bias):
    scaled = (A.double() @ W.double().t()) * sA.double()[:, None] * sW.double()  # (the sums are exact in 64 bits)
    want = scaled if bias is None else scaled + bias.double()
    # the sum's conversion, two products, the bias
    assert_near(got, want, 4 * U * (scaled.abs() + (0 if bias is None else bias.double().abs())))


SHAPES = [(1, 1, 1), (1, 17, 5), (2, 16, 15), (3, 100, 16), (16, 64, 64), (17, 33, 100), (31, 70, 1000), (33, 129, 63), (64, 200, 257), (65, 1, 1),
          (65, 127, 17), (66, 300, 128), (100, 1000, 129), (128, 128, 128), (129, 255, 400), (200, 384, 1024), (257, 513, 640), (300, 200, 4096), (1, 4096, 4096),
          (5, 1000, 8191), (64, 5000, 300), (1000, 1000, 1000), (256, 256, 4096), (512, 768, 2048), (1000, 40, 20000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(seed, M, N, K, dtype):
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    for b in (None, bias):
        _check(q.qnn_int8_gemm(A, sA, W, sW, b, dtype=dtype), A, sA, W, sW, b)


@pytest.mark.parametrize("M,N,K,pad_a,pad_w,offset", [(5, 70, 64, 1, 0, 0), (5, 70, 100, 28, 28, 16), (40, 70, 100, 3, 5, 1), (200, 300, 256, 16, 16, 16), (200, 300, 256, 1, 16, 0),
                                                      (200, 300, 256, 16, 7, 0), (200, 300, 250, 6, 6, 0), (200, 300, 250, 6, 6, 3), (300, 257, 1000, 24, 24, 0),
                                                      (600, 600, 1024, 0, 0, 8), (600, 600, 1024, 64, 192, 32)])
def test_strides(seed, M, N, K, pad_a, pad_w, offset):
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    _, a = placed(A, pad_a, offset, 101)
    _, w = placed(W, pad_w, offset, 99)
    for pad_o, at in ((0, 0), (1, 1), (8, 8), (16, 0)):
        for dtype in TYPES:
            whole, out = placed(torch.zeros(M, N, dtype=dtype, device="cuda"), pad_o, at, 7.0)
            assert q.qnn_int8_gemm(a, sA, w, sW, bias, out) is out
            _check(out, A, sA, W, sW, bias)
            assert untouched(whole, out, 7.0)


@pytest.mark.parametrize("M,N", [(2, 3), (70, 20), (256, 256)])
def test_largest_sums(M, N):
    """131071 products of -128 and -128: 2^31 - 2^14."""
    import paper_1609_07061_amd as q

    K = 131071
    A, W = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    one = lambda n: torch.ones(n, device="cuda")
    assert (q.qnn_int8_gemm(A, one(M), W, one(N), dtype=torch.float32) == float(K * 16384)).all()
    W.fill_(127)
    assert (q.qnn_int8_gemm(A, one(M), W, one(N), dtype=torch.float32) == torch.tensor(-float(K * 128 * 127))).all()


@pytest.mark.parametrize("M", [4, 100, 300])
def test_scales_without_a_value(seed, M):
    """A row or channel whose scale is NaN or infinite, or zero, has that effect on its own outputs only."""
    import paper_1609_07061_amd as q

    A, sA, W, sW, _ = _operands(seed, M, 300, 512)
    sA[1], sA[2], sW[5] = float("nan"), 0.0, float("nan")
    got = q.qnn_int8_gemm(A, sA, W, sW, dtype=torch.float32)
    assert torch.isnan(got[1]).all() and torch.isnan(got[:, 5]).all()
    rows, cols = [m for m in range(M) if m != 1], [n for n in range(300) if n != 5]
    assert (got[2, cols] == 0).all()
    _check(got[rows][:, cols], A[rows], sA[rows], W[cols], sW[cols], None)


def test_offsets_beyond_32_bits(seed):
    """Rows that lie more than 4 GiB apart."""
    import paper_1609_07061_amd as q

    K, pitch = 256, (1 << 31) + 64
    whole = torch.zeros(2 * pitch + K, dtype=torch.int8, device="cuda")
    A = whole.as_strided((3, K), (pitch, 1))
    g = generator(seed, 77)
    A.copy_(codes_of(g, 3, K))
    W, sW = codes_of(g, 40, K), normal(g, 40)
    sA = torch.ones(3, device="cuda")
    _check(q.qnn_int8_gemm(A, sA, W, sW, dtype=torch.float32), A.contiguous(), sA, W, sW, None)
    B = codes_of(g, 100, K)
    _check(q.qnn_int8_gemm(B, torch.ones(100, device="cuda"), A, sA, dtype=torch.float32), B, torch.ones(100, device="cuda"), A.contiguous(), sA, None)


def test_empty():
    import paper_1609_07061_amd as q

    z = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda")
    f = lambda n: torch.zeros(n, device="cuda")
    assert q.qnn_int8_gemm(z(0, 8), f(0), z(5, 8), f(5)).shape == (0, 5)
    assert q.qnn_int8_gemm(z(3, 8), f(3), z(0, 8), f(0)).shape == (3, 0)


@pytest.mark.parametrize("M,N,K", [(1, 512, 512), (300, 512, 1024)])
def test_other_stream_and_graph(seed, M, N, K):
    """The current stream is the one used; a captured call replays on new inputs."""
    import paper_1609_07061_amd as q

    A, sA, W, sW, bias = _operands(seed, M, N, K)
    out = torch.zeros(M, N, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        q.qnn_int8_gemm(A, sA, W, sW, bias, out)
    s.synchronize()
    _check(out, A, sA, W, sW, bias)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.qnn_int8_gemm(A, sA, W, sW, bias, out)
    for i in range(3):
        A.copy_(codes_of(generator(seed, i), M, K))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, q.qnn_int8_gemm(A, sA, W, sW, bias, dtype=torch.float32))
