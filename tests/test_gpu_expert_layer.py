"""A layer of routed experts behind a compressed router (paper_1711_00244_amd.experts): each of its steps against the plain fp64 forms (mx_ref),
and the whole as one call, recorded call and refused call."""
import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_1711_00244_amd as cl
from paper_1711_00244_amd import experts as ex

pytestmark = pytest.mark.gpu


def values(Q):
    return ref.values(Q.codes.cpu().numpy(), Q.scales.cpu().numpy(), Q.K)


def tokens_of(T, width, seed=1):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((T, width), dtype=np.float32)).cuda()


@pytest.mark.parametrize("T,experts,width,hidden,k,shared", [(1, 8, 130, 34, 2, True), (3, 16, 256, 40, 4, False), (70, 16, 200, 66, 4, True), (400, 5, 136, 32, 1, True)])
def test_layer_against_its_steps(T, experts, width, hidden, k, shared):
    layer = ex.synthetic(experts, width, hidden, k, shared=shared, seed=T, score="sigmoid", scale=1.5)
    X = tokens_of(T, width)
    Y = layer.forward(X)
    chosen, weights = layer.route(X)

    # the router: the dense matrix that the compressed layer stands for
    dense = cl.decode_layer(layer.router)[3].double().cpu().numpy()
    logits = X.double().cpu().numpy() @ dense.T
    e, w, sure = ref.route(logits, None, k, "sigmoid", 1, 1, "max", True, 1.5, float(np.finfo(np.float32).min))
    # (the logits are sums of up to `width` fp32 products: where two are closer than that, their order is open)
    top = -np.sort(-logits, axis=1)
    sure &= (top[:, :-1] - top[:, 1:] > 1e-4).all(axis=1)
    assert sure.any()
    assert np.array_equal(chosen.cpu().numpy()[sure], e[sure])
    assert np.abs(weights.cpu().numpy() - w)[sure].max() <= 1e-4

    # the experts: both products with the choice that was made
    xq, up, down = ref.quantised(X.cpu().numpy()), values(layer.up), values(layer.down)
    chosen_np = chosen.cpu().numpy()
    hid = cl.mx_experts_forward(layer.up, X, chosen, act="gated")
    ref.assert_within(hid, *ref.experts(xq, up, chosen_np, None, None, "gated", False))
    out, err = ref.experts(ref.quantised(hid.cpu().numpy()), down, chosen_np, weights.cpu().numpy(), None, "none", True)
    if shared:
        first, second = (values(q) for q in layer.shared)
        mid = cl.mx_fc_forward(layer.shared[0], X, act="gated")
        ref.assert_within(mid, *ref.product(xq, first, None, "gated"))
        o, r = ref.product(ref.quantised(mid.cpu().numpy()), second, None, "none")
        # (two values rounded to fp32 before their sum is)
        out, err = out + o, err + r + 2.0 ** -23 * (np.abs(out) + np.abs(o) + err + r)
    ref.assert_within(Y, out, err)


@pytest.mark.parametrize("T", [1, 90])
def test_layer_recorded(T):
    layer = ex.synthetic(16, 256, 64, 2, seed=5)
    X = tokens_of(T, 256)
    layer.forward(X)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = layer.forward(X)
    for seed in (2, 3, 4):
        X.copy_(tokens_of(T, 256, seed))
        graph.replay()
        got = Y.clone()
        assert torch.equal(got, layer.forward(X))


def test_layer_of_no_tokens():
    layer = ex.synthetic(8, 128, 32, 2)
    assert layer.forward(torch.empty((0, 128), device="cuda")).shape == (0, 128)


def test_layer_refuses_matrices_that_do_not_fit():
    good = ex.synthetic(8, 128, 32, 2)
    other = ex.synthetic(8, 160, 32, 2)
    with pytest.raises(ValueError):
        ex.ExpertLayer(good.router, other.up, other.down, 2)
    with pytest.raises(ValueError):
        ex.ExpertLayer(good.router, good.up, other.down, 2)
    with pytest.raises(ValueError):
        ex.ExpertLayer(good.router, good.up, good.down, 2, other.shared)
    with pytest.raises(cl.CLError):
        ex.ExpertLayer(good.router, good.up, good.down, 9).forward(tokens_of(2, 128))
