"""Weights of chosen experts whose scores are tiny - a bias brings experts in that softmax gives almost nothing, or every logistic score is small - are
quotients of scores, and those are ordinary numbers also where the scores are below fp32's smallest."""
import numpy as np
import pytest
import torch

import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu

# experts, groups, k: sixteen lanes to a token, sixty-four
SIZES = [(8, 1, 3), (64, 4, 8), (200, 1, 5), (256, 8, 16), (500, 1, 2), (700, 1, 4), (300, 20, 6), (96, 2, 20)]


def expected(x, chosen):
    """exp(x_j) / sum of exp over the chosen, fp64."""
    v = np.take_along_axis(x, chosen, 1)
    v = np.exp(v - v.max(1, keepdims=True))
    return v / v.sum(1, keepdims=True)


# fp32: one part in 2^24 for each of up to 20 additions, a few for exponential and division, and for the difference of two logits below 512, exact to
# 2^-15: 2e-5 relative of the largest weight holds them all with room to spare
GATE = 2e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("E,groups,k", SIZES)
@pytest.mark.parametrize("depth", [30, 60, 90, 100, 120, 400])
def test_softmax_with_a_bias(dtype, E, groups, k, depth):
    rng = np.random.default_rng(E + depth)
    T = 9
    # expert 0 has all of the softmax and a bias that keeps it out; the others are `depth` below, in quarters, in an order that the bias gives
    x = -depth - rng.integers(0, 12, (T, E)) / 4.0
    x[:, 0] = 0.0
    bias = np.concatenate([[-8.0], rng.permutation(E - 1) / E + 1.0]).astype(np.float32)
    xd = torch.from_numpy(x).to("cuda", dtype)
    e, w = cl.route_experts(xd, k, bias=torch.from_numpy(bias).cuda(), groups=groups)
    e, w = e.cpu().numpy(), w.cpu().numpy()
    if groups == 1:
        assert np.array_equal(e, np.broadcast_to(np.argsort(-bias, kind="stable")[:k], (T, k)))
    assert (e > 0).all()
    assert np.abs(w - expected(xd.double().cpu().numpy(), e)).max() <= GATE


@pytest.mark.parametrize("E,groups,k", SIZES)
@pytest.mark.parametrize("depth", [30, 60, 85, 100, 120, 400])
def test_logistic(E, groups, k, depth):
    rng = np.random.default_rng(E + depth)
    T = 9
    x = -depth - np.stack([rng.permutation(E) for _ in range(T)]) * (8.0 / E)
    xd = torch.from_numpy(x).to("cuda", torch.float32)
    bias = torch.from_numpy((rng.permutation(E) / E).astype(np.float32)).cuda()
    for b in (None, bias) if groups == 1 else (bias,):       # (group scores below fp32's smallest are equal)
        e, w = cl.route_experts(xd, k, bias=b, score="sigmoid", groups=groups, scale=2.5)
        e = e.cpu().numpy()
        assert (e >= 0).all()
        assert np.abs(w.cpu().numpy() / 2.5 - expected(xd.double().cpu().numpy(), e)).max() <= GATE


def test_what_stays_zero():
    x = torch.full((4, 64), -300.0, device="cuda")
    x[0, :] = -torch.inf                                     # nobody left
    x[1, 3] = torch.inf                                      # the others have nothing at all beside it
    x[2, 5:] = -torch.inf                                    # fewer than k left
    x[3, 0] = 0.0
    bias = torch.zeros(64, device="cuda")
    bias[3] = -torch.inf
    bias[0] = -5.0
    e, w = cl.route_experts(x, 4, bias=bias)
    assert (e[0] == -1).all() and (w[0] == 0).all()
    assert not bool((e[1] == 3).any()) and (w[1] == 0).all()
    assert e[2].tolist() == [1, 2, 4, 0] and bool(w.isfinite().all())
    assert e[3].tolist() == [1, 2, 4, 5] and w[3].tolist() == [0.25] * 4
    # the scores themselves, without the quotient, round to zero
    assert (cl.route_experts(x, 4, bias=bias, renormalize=False)[1][3] == 0).all()
