"""The choice of experts for more tokens than one launch has threads for: sixteen lanes to a token and sixty-four."""
import pytest
import torch

import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,groups", [((1 << 28) + 19, 2, 1), ((1 << 26) + 19, 17, 17)])
def test_more_tokens_than_a_launch_holds(T, E, groups):
    x = torch.zeros((T, E), dtype=torch.bfloat16, device="cuda")
    x[:, 1] = -1.0
    # the tokens around the ends of pieces, the first and the last choose the other one
    other = torch.tensor([0, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, (1 << 27) - 1, 1 << 27, 1 << 28, T - 1], device="cuda").clamp_max(T - 1)
    x[other, 1] = 1.0
    e, w = cl.route_experts(x, 1, groups=groups)
    assert int(e.sum()) == len(other.unique()) and bool((e[other] == 1).all()) and bool((e >= 0).all())
    assert bool((w == 1).all())
