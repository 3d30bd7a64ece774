"""examples/int8_feed_forward.py: what it computes, by autograd on the same values, and that it learns and replays."""
import importlib.util
import os

import pytest
import torch

from int8_testlib import silu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "int8_feed_forward.py")
    spec = importlib.util.spec_from_file_location("int8_feed_forward", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("rows", [1, 37])
def test_gradients(example, rows):
    """Against autograd of the unquantized path in float64: codes are within half a step of 1/127 of the row's largest value, and bf16 keeps 8 bits; the
    gradients of a path this short agree to a few per cent (the bound, 0.1 of the largest, is five times the 2 % that half a step of both factors gives)."""
    layer = example.FeedForward(128, 192, 5)
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, res, grad = (torch.randn(rows, 128, device="cuda", generator=g).bfloat16() for _ in range(3))
    y, h, kept = layer.forward(x, res)
    got = layer.backward(grad, kept)
    leaves = [t.double().requires_grad_() for t in (h, layer.gamma, layer.w1, layer.w2)]
    hh, gamma, w1, w2 = leaves
    u = (hh / (hh.square().mean(dim=1, keepdim=True) + example.EPS).sqrt() * gamma) @ w1.t()
    out = (silu(u[:, :192]) * u[:, 192:]) @ w2.t()
    assert (y.double() - out).abs().max() <= 0.1 * out.abs().max()
    want = torch.autograd.grad(((out + hh) * grad.double()).sum(), leaves)
    for a, b in zip(got, want):
        assert a.shape == b.shape and (a.double() - b).norm() <= 0.1 * b.norm()


def test_training_learns(example):
    errors = example.train(steps=30)
    assert errors[-1] < 0.5 * errors[0]


@pytest.mark.parametrize("tokens", [1, 16])
def test_serving_replays(example, tokens):
    out, want, _ = example.serve(tokens)
    assert torch.equal(out, want) and bool(torch.isfinite(out).all()) and bool((out != 0).any())
