"""mx_fc_forward's two ways to name what follows the product agree, or the call is refused: relu=True beside another act is not dropped."""
from types import SimpleNamespace

import pytest
import torch

import paper_1711_00244_amd as cl


@pytest.mark.parametrize("act", ["none", "gated"])
def test_relu_beside_another_act(act):
    W = SimpleNamespace(codes=torch.zeros((4, 64), dtype=torch.uint8), K=64)         # (refused before anything of it is looked at)
    with pytest.raises(ValueError, match="relu"):
        cl.mx_fc_forward(W, None, relu=True, act=act)


@pytest.mark.gpu
def test_what_agrees():
    W, x = cl.mx_quantize(torch.randn((6, 64), device="cuda")), torch.randn((5, 64), device="cuda")
    y = cl.mx_fc_forward(W, x)
    assert bool((y < 0).any())
    for how in (dict(relu=True), dict(act="relu"), dict(relu=True, act="relu")):
        assert torch.equal(cl.mx_fc_forward(W, x, **how), y.clamp_min(0))
    for how in (dict(relu=False, act="none"), dict(act=None)):
        assert torch.equal(cl.mx_fc_forward(W, x, **how), y)
