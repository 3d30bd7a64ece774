"""Calls on int8 codes with more workgroups than one dimension of a launch takes (2^32 threads)."""
import pytest
import torch

from int8_testlib import codes_of, generator, normal

pytestmark = pytest.mark.gpu


def _all_equal(got, want):
    """Whether `got` is `want` again and again, part by part."""
    whole = got.shape[0] // want.shape[0]
    parts = torch.split(got[: whole * want.shape[0]].unflatten(0, (whole, want.shape[0])), max(1, whole // 16))
    return all(bool((p == want[None]).all()) for p in parts) and torch.equal(got[whole * want.shape[0] :], want[: got.shape[0] % want.shape[0]])


@pytest.mark.parametrize("K", [1, 9])
def test_rows(seed, K):
    """2^26 rows and more, of a wave each."""
    import paper_1609_07061_amd as q

    few, rows = 4099, (1 << 26) + 4321
    base = normal(generator(seed, K, 8), few, 2 * K).half()
    x = base.repeat(rows // few + 1, 1)[:rows]
    gamma = (1 + normal(generator(seed, 9), K) / 4).half()
    codes, scale, _ = q.qnn_rms_norm_quant(x[:, :K], gamma, 1e-5)
    want = q.qnn_rms_norm_quant(base[:, :K], gamma, 1e-5)
    assert _all_equal(codes, want[0]) and _all_equal(scale, want[1])
    q.qnn_silu_gate_quant(x[:, :K], x[:, K:], codes, scale)
    want = q.qnn_silu_gate_quant(base[:, :K], base[:, K:])
    assert _all_equal(codes, want[0]) and _all_equal(scale, want[1])


def test_products_of_short_rows():
    """More than 2^31 outputs in tiles of 16 x 16 on 512 threads each."""
    import paper_1609_07061_amd as q

    g, n, times = torch.Generator(device="cuda").manual_seed(5), 64, 725
    A, W, sA, sW = codes_of(g, n, 3), codes_of(g, n, 3), normal(g, n), normal(g, n) * 0.01
    want = q.qnn_int8_gemm(A, sA, W, sW, dtype=torch.float16)
    assert ((want.double() - (A.double() @ W.double().t()) * sA.double()[:, None] * sW.double()).abs() <= 2.0 ** -10 * want.double().abs() + 2.0 ** -24).all()
    got = q.qnn_int8_gemm(A.repeat(times, 1), sA.repeat(times), W.repeat(times, 1), sW.repeat(times), dtype=torch.float16)
    assert _all_equal(got, want.repeat(1, times))


@pytest.mark.parametrize("K", [16, 17])
def test_products_of_many_rows(K):
    """2^29 rows and more, in tiles of 64 x 16 on 512 threads each."""
    import paper_1609_07061_amd as q

    g, few, rows = torch.Generator(device="cuda").manual_seed(K), 4099, (1 << 29) + 4321
    A, W, sA, sW = codes_of(g, few, K), codes_of(g, 3, K), normal(g, few), normal(g, 3) * 0.01
    want = q.qnn_int8_gemm(A, sA, W, sW, dtype=torch.float16)
    assert ((want.double() - (A.double() @ W.double().t()) * sA.double()[:, None] * sW.double()).abs() <= 2.0 ** -10 * want.double().abs() + 2.0 ** -24).all()
    times = rows // few + 1
    got = q.qnn_int8_gemm(A.repeat(times, 1)[:rows], sA.repeat(times)[:rows], W, sW, dtype=torch.float16)
    assert _all_equal(got, want)
