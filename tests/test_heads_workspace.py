"""The workspace of the gradient of norm and rotation: one that is made for the most tokens serves all calls."""
import pytest
import torch


@pytest.mark.parametrize("heads_q,heads_k", [(1, 1), (32, 8), (0, 4), (4, 0), (65535, 1), (7, 9)])
def test_never_less_for_more(heads_q, heads_k):
    import paper_1609_07061_amd as q

    sizes = [q.qnn_qk_norm_rotate_backward_workspace_bytes(t, heads_q, heads_k, 64) for t in [*range(1, 5000), 8192, 100000, 1 << 30]]
    assert sizes[0] > 0 and sizes == sorted(sizes) and sizes[-1] <= 1025 * 64 * 4


@pytest.mark.gpu
def test_one_for_all_calls(seed):
    from attention_testlib import Rotation, heads_of
    import paper_1609_07061_amd as q

    D = 64
    gamma = torch.ones(D, device="cuda")
    ws = torch.empty(q.qnn_qk_norm_rotate_backward_workspace_bytes(5000, 4, 2, D), dtype=torch.uint8, device="cuda")
    for T in (5000, 4096, 2731, 700, 512, 511, 40, 1):
        rotation = Rotation(seed, T, D)
        x, k, dx, dk = (heads_of(seed + i, T, H, D, torch.bfloat16) for i, H in enumerate((4, 2, 4, 2)))
        ws.fill_(255)
        got = q.qnn_qk_norm_rotate_backward(dx, dk, x, k, gamma, gamma, 1e-6, *rotation.args, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(got, q.qnn_qk_norm_rotate_backward(dx, dk, x, k, gamma, gamma, 1e-6, *rotation.args)))
