"""The 256 x 256 tile of the 8-bit products with outputs in fp16: one step of k to a tile, several, more tiles than compute units, k in shares, with and without gates and biases."""
import pytest
import torch

import paper_1711_00244_amd as cl
from test_gpu_f8_forms import F8, F16, check, draw, product, same, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("splits,B,M,K,x_type,act", [(1, 5537, 1166, 35, F16, "gated"), (1, 4500, 1300, 900, F16, "gated"), (1, 5100, 2470, 900, F16, "none"), (1, 5000, 2500, 130, F8, "relu"),
                                                     (8, 4704, 131, 24334, F16, "none")])
def test_tile_256_in_fp16(splits, B, M, K, x_type, act):
    W, X, bias = draw(B, M, K, act == "gated", B + M, F16)
    if x_type == F8:
        X = cl.f8_quantize(X)
    assert cl.f8_fc_resolved_form(W, B, x_type, act, F16) == ("tile 256", splits)
    x = wide(X if x_type == F8 else cl.f8_quantize(X))
    for b in (None, bias):
        want, err = product(x, wide(W), b, act, True)
        y = cl.f8_fc_forward(W, X, b, act=act, dtype=F16)
        assert y.dtype == F16
        check(y, want, err, (splits, b is None))
        assert same(y, cl.f8_fc_forward(W, X, b, act=act, dtype=F16))
