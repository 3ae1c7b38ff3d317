"""The choice of experts, the lists of their tokens, and their products, against plain fp64 forms (mx_ref)."""
import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


def route_both(x, k, bias=None, **how):
    kw = dict(score="softmax", groups=1, groups_kept=None, group_score="max", renormalize=True, scale=1.0)
    kw.update(how)
    e, w = cl.route_experts(x, k, bias=bias, **kw)
    b = None if bias is None else bias.double().cpu().numpy()
    kept = kw["groups"] if kw["groups_kept"] is None else kw["groups_kept"]
    we, ww, sure = ref.route(x.double().cpu().numpy(), b, k, kw["score"], kw["groups"], kept, kw["group_score"], kw["renormalize"], kw["scale"],
                             float(torch.finfo(x.dtype).min))
    assert sure.mean() >= 0.5                                # (the others hang on an order that fp32 does not have to give)
    assert np.array_equal(e.cpu().numpy()[sure], we[sure]), how
    # exponential, division, sums of up to 1024 scores and of k, each within a few units of the last place
    assert np.abs(w.cpu().numpy() - ww)[sure].max(initial=0.0) <= 2e-5 * np.abs(ww).max(initial=1e-30), how
    return e, w


def logits(rng, T, E, dtype, step=None):
    """Values on a grid (a permutation of it per token where `step` is None), so that keys are equal or well apart."""
    if step is None:
        x = np.stack([rng.permutation(E) for _ in range(T)]) * (8.0 / E) - 4 if T else np.zeros((0, E))
    else:
        x = np.round(rng.standard_normal((T, E)) / step) * step
    return torch.from_numpy(x).to("cuda", dtype)


# tokens, experts, k
SIZES = [(1, 1, 1), (1, 8, 2), (3, 64, 8), (5, 7, 7), (70, 60, 6), (33, 65, 17), (9, 128, 32), (20, 200, 8), (130, 256, 8), (4, 300, 9), (11, 1024, 4), (1000, 16, 1)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route(T, E, k, score):
    rng = np.random.default_rng(T + E + k)
    for dtype in ref.DTYPES:
        for step in (None, 0.5):                             # 0.5: many equal logits, of which the lower expert comes first
            if step is None and dtype is torch.bfloat16 and E > 200:
                continue                                     # (the grid is finer than the type)
            x = logits(rng, T, E, dtype, step)
            route_both(x, k, score=score, renormalize=step is None, scale=1.0 if step else 2.5)


@pytest.mark.parametrize("E,groups,kept,k", [(8, 2, 1, 3), (24, 4, 2, 5), (64, 8, 4, 8), (256, 8, 4, 8), (60, 3, 3, 2), (64, 64, 9, 9), (96, 2, 1, 20), (500, 20, 7, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_route_in_groups(E, groups, kept, k, score, group_score):
    rng = np.random.default_rng(E + k)
    T = 40
    for bias in (None, torch.from_numpy((rng.integers(-40, 41, E) * 0.015625).astype(np.float32)).cuda()):
        x = logits(rng, T, E, torch.float32)
        route_both(x, k, bias=bias, score=score, groups=groups, groups_kept=kept, group_score=group_score)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("E,groups,kept,k", [(64, 1, 1, 8), (40, 4, 2, 6), (256, 8, 4, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masks(dtype, E, groups, kept, k, score):
    rng = np.random.default_rng(E)
    x = logits(rng, 12, E, dtype)
    low = torch.finfo(dtype).min
    x[0, :] = -torch.inf                                     # nothing left
    x[1, :] = low
    x[2, :] = torch.nan
    x[3, : E - 2] = -torch.inf                               # fewer than k left
    x[4, 1:] = low
    x[5, ::2] = -torch.inf
    x[6, 3] = torch.nan
    x[7, 5] = torch.inf
    x[8, 5], x[8, 9] = torch.inf, torch.inf
    bias = torch.zeros(E, device="cuda")
    e, w = route_both(x, k, score=score, groups=groups, groups_kept=kept, group_score="top2")
    assert (e[:3] == -1).all() and (w[:3] == 0).all()
    assert bool(w.isfinite().all())
    # a bias cannot bring a masked logit back, and can mask by itself
    bias[0], bias[1] = 5.0, -torch.inf
    x[9, 0] = -torch.inf
    e, w = route_both(x, k, bias=bias, score=score, groups=groups, groups_kept=kept, group_score="max")
    assert not bool((e == 1).any()) and not bool((e[9] == 0).any())


def test_route_rows_at_a_distance_and_none():
    rng = np.random.default_rng(3)
    buf = logits(rng, 9, 70, torch.float32)
    route_both(buf[:, 3:67], 4)
    e, w = cl.route_experts(torch.empty((0, 64), device="cuda"), 4)
    assert e.shape == w.shape == (0, 4)


@pytest.mark.parametrize("T,k,E", [(0, 2, 4), (1, 1, 1), (1, 8, 64), (5, 3, 2), (100, 4, 16), (1025, 1, 7), (700, 8, 300), (3000, 6, 1024)])
def test_lists(T, k, E):
    rng = np.random.default_rng(T + E)
    e = rng.integers(-1, E + 1, (T, k)).astype(np.int32)     # -1 and E: none
    e[rng.random((T, k)) < 0.3] = min(1, E - 1)              # a busy one
    L = cl.expert_lists(torch.from_numpy(e).cuda(), E)
    flat = np.where((e < 0) | (e >= E), E, e).reshape(-1)
    want = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1))])
    assert np.array_equal(L.offsets.cpu().numpy(), want)


# tokens, experts, k, rows, K
SHAPES = [(1, 1, 1, 16, 128), (1, 8, 2, 33, 100), (2, 64, 8, 48, 513), (7, 4, 3, 100, 300), (40, 6, 2, 130, 640), (100, 24, 3, 50, 410), (300, 5, 2, 96, 256),
          (600, 3, 1, 260, 384), (513, 16, 4, 70, 200)]


def case(rng, T, E, k, M, K, dtype, x_rows):
    x = torch.from_numpy(rng.standard_normal((x_rows, K))).to("cuda", dtype)
    w = cl.mx_quantize(torch.from_numpy((rng.standard_normal((E, M, K)) * 0.05).astype(np.float32)).cuda())
    e = rng.integers(0, E, (T, k)).astype(np.int32)
    e[rng.random((T, k)) < 0.1] = -1
    e[rng.random((T, k)) < 0.02] = E + 3
    wt = rng.random((T, k)).astype(np.float32)
    bias = rng.standard_normal((E, M)).astype(np.float32)
    return x, w, e, wt, bias, ref.quantised(x.double().cpu().numpy()), ref.values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), K)


@pytest.mark.parametrize("T,E,k,M,K", SHAPES)
def test_experts(T, E, k, M, K):
    rng = np.random.default_rng(T + M)
    for dtype in ref.DTYPES:
        x, w, e, wt, bias, xq, wq = case(rng, T, E, k, M, K, dtype, T)
        ed, wd, bd = torch.from_numpy(e).cuda(), torch.from_numpy(wt).cuda(), torch.from_numpy(bias).cuda()
        lists = cl.expert_lists(ed, E)
        for weights, b, act in ((wt, None, "none"), (None, bias, "relu"), (wt, bias, "relu")):
            y = cl.mx_experts_forward(w, x, ed, None if weights is None else wd, None if b is None else bd, act=act)
            assert y.dtype == dtype
            ref.assert_within(y, *ref.experts(xq, wq, e, weights, b, act, False), (T, E, k, M, K, dtype, act))
            z = cl.mx_experts_forward(w, cl.mx_quantize(x), ed, None if weights is None else wd, None if b is None else bd, act=act, lists=lists, dtype=dtype)
            assert torch.equal(y, z)


@pytest.mark.parametrize("T,E,k,M,K", [(1, 8, 2, 34, 100), (3, 5, 2, 100, 300), (90, 7, 3, 66, 200), (700, 4, 1, 130, 130)])
def test_gated_experts_and_rows_per_pair(T, E, k, M, K):
    rng = np.random.default_rng(T * M)
    x, w, e, wt, bias, xq, wq = case(rng, T, E, k, M, K, torch.float32, T)
    ed, wd, bd = torch.from_numpy(e).cuda(), torch.from_numpy(wt).cuda(), torch.from_numpy(bias).cuda()
    y = cl.mx_experts_forward(w, x, ed, None, bd, act="gated")
    assert y.shape == (T * k, M // 2)
    ref.assert_within(y, *ref.experts(xq, wq, e, None, bias, "gated", False))
    x, w, e, wt, bias, xq, wq = case(rng, T, E, k, M, K, torch.bfloat16, T * k)
    ed, wd = torch.from_numpy(e).cuda(), torch.from_numpy(wt).cuda()
    for weights in (None, wt):
        y = cl.mx_experts_forward(w, x, ed, None if weights is None else wd, x_per_pair=True)
        ref.assert_within(y, *ref.experts(xq, wq, e, weights, None, "none", True))


@pytest.mark.parametrize("T", [1, 50, 800])
def test_all_tokens_to_one_expert_and_none_to_any(T):
    rng = np.random.default_rng(T)
    x, w, e, wt, bias, xq, wq = case(rng, T, 9, 2, 40, 130, torch.float32, T)
    wd, bd = torch.from_numpy(wt).cuda(), torch.from_numpy(bias).cuda()
    e[:] = 6
    ed = torch.from_numpy(e).cuda()
    ref.assert_within(cl.mx_experts_forward(w, x, ed, wd), *ref.experts(xq, wq, e, wt, None, "none", False))
    ed.fill_(-1)
    for weights in (None, wd):
        y = cl.mx_experts_forward(w, x, ed, weights, bd, out=torch.full((T if weights is not None else 2 * T, 40), 5.0, device="cuda"))
        assert bool((y == 0).all())


def test_what_is_not_finite_stays_with_its_token():
    rng = np.random.default_rng(0)
    T = 60
    x, w, e, wt, _, _, _ = case(rng, T, 6, 2, 50, 200, torch.float32, T)
    e = np.where((e < 0) | (e >= 6), 0, e)
    ed, wd = torch.from_numpy(e).cuda(), torch.from_numpy(wt).cuda()
    y = cl.mx_experts_forward(w, x, ed, wd)
    x[7, 100] = float("nan")
    z = cl.mx_experts_forward(w, x, ed, wd)
    rest = torch.arange(T, device="cuda") != 7
    assert z[7].isnan().all() and torch.equal(z[rest], y[rest])


@pytest.mark.parametrize("T", [2, 300])
def test_captured(T):
    rng = np.random.default_rng(T)
    x, w, e, wt, _, _, _ = case(rng, T, 6, 2, 50, 200, torch.float32, T)
    ed, wd = torch.from_numpy(e).cuda(), torch.from_numpy(wt).cuda()
    out = cl.mx_experts_forward(w, x, ed, wd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cl.mx_experts_forward(w, x, ed, wd, out=out)
    for i in range(3):
        x.copy_(torch.roll(x, 1, 0) * 1.5)
        ed.copy_(torch.roll(ed, 1, 0))
        out.zero_()
        eager = cl.mx_experts_forward(w, x, ed, wd)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_refusals_of_the_binding():
    x = torch.ones((4, 64), device="cuda")
    w = cl.mx_quantize(torch.ones((3, 8, 64), device="cuda"))
    e = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    for bad in (e.long(), e[:3], e.t(), e.cpu()):
        with pytest.raises(ValueError):
            cl.mx_experts_forward(w, x, bad)
    with pytest.raises(ValueError):
        cl.mx_experts_forward(cl.mx_quantize(x), x, e)
    with pytest.raises(ValueError):
        cl.mx_experts_forward(w, x, e, weights=torch.ones((4, 3), device="cuda"))
    with pytest.raises(ValueError):
        cl.mx_experts_forward(w, x, e, bias=torch.ones(8, device="cuda"))
    with pytest.raises(ValueError):
        cl.mx_experts_forward(w, x, e, lists=cl.expert_lists(e, 4))
    with pytest.raises(ValueError):
        cl.mx_experts_forward(w, x, e, x_per_pair=True)
    with pytest.raises(cl.CLError):
        cl.mx_experts_forward(w, torch.ones((100000, 64), device="cuda"), torch.zeros((100000, 2), dtype=torch.int32, device="cuda"),
                              workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    for kw in (dict(k=0), dict(k=65), dict(k=2, groups=3), dict(k=2, groups=4, groups_kept=5), dict(k=20, groups=4, groups_kept=1)):
        with pytest.raises(cl.CLError):
            cl.route_experts(x, **kw)
    for kw in (dict(score="relu"), dict(group_score="mean"), dict(bias=torch.ones(3, device="cuda"))):
        with pytest.raises(ValueError):
            cl.route_experts(x, 2, **kw)
