"""How examples/int8_feed_forward.py lays weights out as codes: the definition of qnn_silu_gate_quant's codes, channels without a value too.  Nothing is launched here."""
import importlib.util
import math
import os

import pytest
import torch


@pytest.fixture(scope="module")
def codes_of_rows():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "int8_feed_forward.py")
    spec = importlib.util.spec_from_file_location("int8_feed_forward", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module.codes_of_rows


@pytest.mark.parametrize("shape", [(7, 40), (3, 7, 40)])
def test_codes_of_rows(codes_of_rows, shape):
    w = torch.randn(*shape, generator=torch.Generator().manual_seed(1))
    w[..., 1, :] = 0
    w[..., 2, 5] = math.nan
    w[..., 3, 6] = math.inf
    w[..., 4, :] = 0
    w[..., 4, 9] = 1e-44  # its scale is 0 in fp32
    codes, scale = codes_of_rows(w)
    assert codes.dtype == torch.int8 and codes.shape == w.shape and scale.dtype == torch.float32 and scale.shape == w.shape[:-1]
    assert (scale[..., 1] == 0).all() and torch.isnan(scale[..., 2:4]).all() and (codes[..., 1:5, :] == 0).all() and (scale[..., 4] == 0).all()
    y = w[..., [0, 5, 6], :].double()
    top = y.abs().amax(dim=-1, keepdim=True)
    assert torch.allclose(scale[..., [0, 5, 6]].double(), top[..., 0] / 127, rtol=2.0 ** -23, atol=0)
    assert ((codes[..., [0, 5, 6], :].double() - y * 127 / top).abs() <= 0.5 + 127 * 2.0 ** -22).all()
