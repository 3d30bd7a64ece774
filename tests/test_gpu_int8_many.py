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
