"""Heads that are all zero, without an eps: zeros, as in the norm of rows.  Tiny values without an eps stay not finite."""
import pytest
import torch

from attention_testlib import Paged, Rotation, heads_of
from int8_testlib import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,pairs,neighbours", [(16, 8, False), (64, 32, True), (80, 24, False), (128, 64, False), (256, 128, True)])
def test_norm_and_rotation(seed, D, pairs, neighbours, dtype):
    import paper_1609_07061_amd as q

    T, H = 5, 6
    rotation = Rotation(seed, T, D, pairs, 1, neighbours)
    x, k = heads_of(seed, T, H, D, dtype), heads_of(seed + 1, T, 2, D, dtype)
    gamma = torch.full((D,), 1.5, device="cuda")
    want = [t.clone() for t in q.qnn_qk_norm_rotate(x, k, gamma, gamma, 0.0, *rotation.args)]
    x[1, 2], x[4], k[3, 0] = 0, 0, -0.0
    tiny = dtype != torch.float16  # (whose least number has a square that fp32 holds)
    if tiny:
        x[0, 3] = 0
        x[0, 3, D - 1] = 1e-30
    got, got_k = q.qnn_qk_norm_rotate(x, k, gamma, gamma, 0.0, *rotation.args)
    assert (got[1, 2] == 0).all() and (got[4] == 0).all() and (got_k[3, 0] == 0).all()
    if tiny:
        assert not torch.isfinite(got[0, 3]).all()
        got[0, 3] = want[0][0, 3]
    got[1, 2], got[4], got_k[3, 0] = want[0][1, 2], want[0][4], want[1][3, 0]
    assert torch.equal(got, want[0]) and torch.equal(got_k, want[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_into_the_cache(seed, dtype):
    """Keys of zeros: codes and scale 0, as the norm of a row gives them, and queries that see them stay finite."""
    import paper_1609_07061_amd as q

    T, D = 20, 64
    p = Paged(seed, [T], [T], 2, D, 16)
    rotation = Rotation(seed, T, D)
    x, k, v = (heads_of(seed + i, T, H, D, dtype) for i, H in enumerate((4, 2, 2)))
    gamma = torch.ones(D, device="cuda", dtype=dtype)
    k[3, 1], k[7], x[5, 2] = 0, 0, 0
    turned = q.qnn_cache_append(*p.args, k, v, gamma, 0.0, *rotation.args, x, gamma)
    page, off, _ = p.places(0)
    codes, scale = p.cache[0][page, :, off], p.cache[1][page, :, off]
    norm_codes, norm_scale = q.qnn_rms_norm_quant(k[7], gamma, 0.0)[:2]
    assert (norm_codes == 0).all() and (norm_scale == 0).all()
    zero = torch.zeros(T, 2, dtype=torch.bool, device="cuda")
    zero[3, 1] = zero[7] = True
    assert (codes[zero] == 0).all() and (scale[zero] == 0).all() and (scale[~zero] > 0).all() and (turned[5, 2] == 0).all()
    assert torch.isfinite(q.qnn_cache_attention(turned, *p.args)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tiny_keys_and_gradients(seed, dtype):
    """Tiny keys without an eps: scale NaN and codes 0, as the norm of a row gives them.  A head of zeros has no gradient then, and all others have theirs."""
    import paper_1609_07061_amd as q

    T, D = 20, 64
    p = Paged(seed, [T], [T], 2, D, 16)
    rotation = Rotation(seed, T, D)
    x, k, v = (heads_of(seed + i, T, H, D, dtype) for i, H in enumerate((4, 2, 2)))
    gamma = torch.ones(D, device="cuda", dtype=dtype)
    k[9, 0] = 0
    k[9, 0, 5] = 1e-30
    q.qnn_cache_append(*p.args, k, v, gamma, 0.0, *rotation.args)
    page, off, _ = p.places(0)
    bad = torch.isnan(p.cache[1][page, :, off])
    assert bad[9, 0] and int(bad.sum()) == 1 and (p.cache[0][page[9], 0, off[9]] == 0).all()
    norm_codes, norm_scale = q.qnn_rms_norm_quant(k[9], gamma, 0.0)[:2]
    assert torch.equal(torch.isnan(norm_scale), bad[9]) and (norm_codes[0] == 0).all()

    dx, dk = heads_of(seed + 5, T, 4, D, dtype), heads_of(seed + 6, T, 2, D, dtype)
    x[5, 2] = 0.25
    k[9, 0] = 0.5
    want = q.qnn_qk_norm_rotate_backward(dx, dk, x, k, gamma, gamma, 0.0, *rotation.args)
    x[5, 2] = 0
    got = q.qnn_qk_norm_rotate_backward(dx, dk, x, k, gamma, gamma, 0.0, *rotation.args)
    assert not torch.isfinite(got[0][5, 2]).any() and not torch.isfinite(got[2]).any()
    got[0][5, 2] = want[0][5, 2]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[3], want[3])
