"""The activation of a gated product, g / (1 + exp(-g)) u, alone: the matrix is zeros, so that every sum is exactly zero and gates and values are the biases."""
import numpy as np
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu
F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, ref.F8

# form, splits, batch, outputs, K, type of X
FORMS = [("few numbers", 1, 5, 333, 1700, F32), ("few", 1, 31, 23, 5068, F32), ("tile 64", 1, 367, 19, 69, F8), ("tile 64", 8, 6, 17, 15527, F32), ("tile 64", 1, 700, 900, 130, F8),
         ("tile 128", 8, 104, 1555, 10491, F8), ("tile 256", 1, 6024, 359, 36, F32)]


def gated(M, K, g, u):
    zeros = cl.f8_quantize(torch.zeros((M, K), device="cuda"), 128)
    return cl.f8_gated(zeros, zeros), torch.from_numpy(np.concatenate([g, u]).astype(np.float32)).cuda()


def inputs(B, K, x_type):
    X = torch.randn((B, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(B))
    return cl.f8_quantize(X) if x_type == F8 else X.to(x_type)


def exact(bias):
    g, u = np.split(bias.double().cpu().numpy(), 2)
    with np.errstate(over="ignore", invalid="ignore"):
        return g / (1 + np.exp(-g)) * u


@pytest.mark.parametrize("form,splits,B,M,K,x_type", FORMS)
def test_gates_in_fp32(form, splits, B, M, K, x_type):
    rng = np.random.default_rng(M)
    g = np.where(rng.random(M) < 0.7, rng.uniform(-86, -4, M), rng.uniform(-4, 90, M))
    u = rng.standard_normal(M) * 2.0 ** rng.integers(-6, 40, M)
    W, bias = gated(M, K, g, u)
    X = inputs(B, K, x_type)
    assert cl.f8_fc_resolved_form(W, B, x_type, "gated", F32) == (form, splits)
    y = cl.f8_fc_forward(W, X, bias, act="gated", dtype=F32)
    assert bool((y == y[0]).all())
    # (exponential and reciprocal: a unit in the last place each, 2 2^-24; the argument's correction, its product, the sum and two products half of one each)
    want = exact(bias)
    off = np.abs(y[0].double().cpu().numpy() - want)
    assert (off <= np.abs(want) * 9 * 2.0 ** -24 * (1 + 2.0 ** -20) + 2.0 ** -149).all(), float((off / np.abs(want)).max() * 2 ** 24)


@pytest.mark.parametrize("form,splits,B,M,K,x_type", FORMS)
def test_8_bit_outputs_have_the_same_gates(form, splits, B, M, K, x_type):
    rng = np.random.default_rng(M + 1)
    W, bias = gated(M, K, rng.uniform(-60, 60, M), rng.standard_normal(M))
    X = inputs(B, K, x_type)
    q, want = cl.f8_fc_forward(W, X, bias, act="gated", dtype=F8), cl.f8_quantize(cl.f8_fc_forward(W, X, bias, act="gated", dtype=F32))
    assert torch.equal(q.scales, want.scales) and torch.equal(q.values.view(torch.uint8), want.values.view(torch.uint8))


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("form,splits,B,M,K,x_type", FORMS)
def test_gates_at_the_ends(form, splits, B, M, K, x_type, out):
    inf, nan, big = np.inf, np.nan, 3.0e38
    g = np.resize([-inf, inf, nan, -big, big, -1e30, -1000.0, -200.0, -89.0, 89.0, 1000.0, 0.0, -0.0, 5.0, 5.0, 5.0, -100.0], M)
    u = np.resize([1.0, 2.0, 1.0, 1.0, 0.5, 1.0, 3.0, 1e30, 1e30, 2.0, -3.0, 7.0, 7.0, inf, nan, -inf, 0.0], M)
    W, bias = gated(M, K, g, u)
    y = cl.f8_fc_forward(W, inputs(B, K, x_type), bias, act="gated", dtype=out)
    assert bool(((y == y[0]) | (y.isnan() & y[0].isnan())).all())
    got = y[0].double().cpu().numpy()
    # (the limit at minus infinity is not taken: minus infinity over infinity.  Gates below -88 are zeros)
    want = exact(bias)
    want[np.isneginf(g)] = nan
    want[(g < -88) & np.isfinite(g)] = 0.0
    want = torch.from_numpy(want).float().to(out).double().numpy()
    ends = ~np.isfinite(want) | (want == 0)
    assert np.array_equal(got[ends], want[ends], equal_nan=True)
    assert (np.abs(got - want)[~ends] <= np.abs(want[~ends]) * {F32: 2.0 ** -20, BF16: 2.0 ** -7, F16: 2.0 ** -10}[out]).all()
