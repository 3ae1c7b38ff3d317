"""Every form of a product with 4-bit matrices, named and checked to be the one that runs, against products that are exact.

Codes are any of the sixteen, scales one of three neighbouring powers of two, drawn for each block: a product of two codes and their scales is a multiple of
1/4 of the smallest scales' product, at most 2304 of them and 110 on average, so that even 25088 of them stay below 2^22 of that unit in absolute sum.  fp32 holds
such sums exactly, in any order and in any parts, and so must every form: a term too many, a term less, a scale of another block or row is seen."""
import pytest
import torch

import paper_1711_00244_amd as cl
from paper_1711_00244_amd import binding

pytestmark = pytest.mark.gpu

GRID = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def blocks(g, shape, K, base=127):
    """-> MxTensor (shape, K) of any codes under scales base .. base + 2 and its values, float64."""
    kb = cl.mx_row_blocks(K)
    q = torch.randint(0, 16, shape + (kb * 32,), generator=g, device="cuda", dtype=torch.uint8)
    q[..., K:] = 0
    scales = torch.randint(base, base + 3, shape + (kb,), generator=g, device="cuda", dtype=torch.uint8)
    v = GRID.cuda()[q.int()] * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    return cl.MxTensor((q[..., 0::2] | q[..., 1::2] << 4).contiguous(), scales, K), v[..., :K].contiguous()


def gen(*seed):
    return torch.Generator(device="cuda").manual_seed(hash(seed) % (1 << 31))


# form, splits, batch, rows, K: loops of 9 steps and more, of every remainder of four, whole and in parts
FC = [("rows", 1, 17, 5755, 1033), ("rows", 1, 17, 2741, 2307), ("rows", 1, 17, 3000, 9216),
      ("tile 64", 1, 33, 7453, 1442), ("tile 64", 1, 6971, 33, 1037), ("tile 64", 1, 7311, 33, 1164), ("tile 64", 1, 33, 7397, 1289),
      ("tile 64", 2, 17, 7488, 3312), ("tile 64", 4, 17, 3960, 6445), ("tile 64", 4, 16, 4096, 25088), ("tile 64", 8, 16, 32, 17068),
      ("tile 128", 1, 9732, 129, 1438), ("tile 128", 1, 8211, 193, 1033), ("tile 128", 1, 8018, 194, 1165), ("tile 128", 1, 10004, 130, 1319),
      ("tile 128", 2, 9541, 65, 3758), ("tile 128", 4, 4258, 67, 10091), ("tile 128", 8, 2049, 66, 14913),
      ("tile 256 x 128", 1, 9460, 392, 1432), ("tile 256 x 128", 1, 9877, 403, 1033), ("tile 256 x 128", 1, 10048, 393, 1157),
      ("tile 256 x 128", 1, 9593, 398, 1348), ("tile 256 x 128", 2, 607, 5398, 25534), ("tile 256 x 128", 4, 132, 5697, 19590),
      ("tile 256", 1, 9444, 770, 1492), ("tile 256", 1, 1050, 7876, 1044), ("tile 256", 1, 8653, 902, 1185), ("tile 256", 1, 9813, 788, 1287),
      ("tile 256", 1, 4096, 4096, 25088), ("tile 256", 2, 8224, 412, 10239), ("tile 256", 4, 8579, 132, 14890), ("tile 256", 8, 5815, 129, 26254)]


@pytest.mark.parametrize("form,splits,B,M,K", FC)
def test_product(form, splits, B, M, K):
    g = gen(B, M, K)
    W, wv = blocks(g, (M,), K)
    X, xv = blocks(g, (B,), K)
    assert cl.mx_fc_resolved_form(W, B) == (form, splits)
    bias = torch.randint(-400, 401, (M,), generator=g, device="cuda").float() / 4
    want = xv @ wv.T
    y = cl.mx_fc_forward(W, X)
    assert y.dtype == torch.float32 and torch.equal(y.double(), want)
    assert torch.equal(cl.mx_fc_forward(W, X, bias, relu=True, dtype=torch.bfloat16), (want + bias.double()).clamp_min(0).to(torch.bfloat16))
    # the values are their own quantisation
    if cl.mx_fc_resolved_form(W, B, torch.bfloat16) == (form, splits):
        assert torch.equal(cl.mx_fc_forward(W, xv.to(torch.bfloat16), dtype=torch.float32), y)


# scales near the ends of what 8 bits hold, on either side
@pytest.mark.parametrize("x_base,w_base", [(0, 250), (250, 0), (5, 249), (127, 12), (12, 127), (250, 40)])
@pytest.mark.parametrize("form,splits,B,M,K", [("few", 1, 3, 70, 900), ("rows", 1, 17, 2741, 2307), ("tile 64", 8, 16, 32, 17068), ("tile 128", 1, 8211, 193, 1033),
                                               ("tile 256", 1, 1050, 7876, 1044)])
def test_far_scales(form, splits, B, M, K, x_base, w_base):
    g = gen(B, M, x_base)
    W, wv = blocks(g, (M,), K, w_base)
    X, xv = blocks(g, (B,), K, x_base)
    want = xv @ wv.T
    assert bool((want.abs()[want != 0] >= 2.0 ** -126).all()) and bool((want.abs() < 2.0 ** 128).all())      # (numbers that fp32 has whole)
    if form == "few":
        assert cl.mx_fc_resolved_form(W, B, torch.float32) == (form, splits)
        assert torch.equal(cl.mx_fc_forward(W, xv.float()).double(), want)
    else:
        assert cl.mx_fc_resolved_form(W, B) == (form, splits)
        assert torch.equal(cl.mx_fc_forward(W, X).double(), want)


def gated(pre):
    """-> silu(g) u and how far off fp32 may be where g and u are exact: a few units of the last place, |g| of them for exp's argument; below
    -88.7, where exp(-g) leaves fp32, all of it, at most 2.6e-37 |u|."""
    gate, up = pre[..., 0::2], pre[..., 1::2]
    out = gate / (1 + torch.exp(-gate)) * up
    return out, (8 + gate.abs()) * 2.0 ** -23 * out.abs() + 3e-37 * up.abs()


@pytest.mark.parametrize("form,splits,B,M,K", [("rows", 1, 17, 5756, 1033), ("tile 64", 1, 6971, 34, 1037), ("tile 64", 2, 17, 7488, 3312), ("tile 64", 8, 16, 32, 17068),
                                               ("tile 128", 1, 8018, 194, 1165), ("tile 128", 8, 2049, 66, 14913), ("tile 256 x 128", 1, 9593, 398, 1348),
                                               ("tile 256", 1, 8653, 902, 1185), ("tile 256", 4, 8579, 132, 14890)])
@pytest.mark.parametrize("base", [118, 122])
def test_gated(form, splits, B, M, K, base):
    g = gen(B, M, base)
    W, wv = blocks(g, (M,), K, base)
    X, xv = blocks(g, (B,), K)
    assert cl.mx_fc_resolved_form(W, B) == (form, splits)
    bias = torch.randint(-400, 401, (M,), generator=g, device="cuda").float() / 64
    for b in (None, bias):
        want, err = gated(xv @ wv.T if b is None else xv @ wv.T + b.double())
        y = cl.mx_fc_forward(W, X, b, act="gated")
        assert y.shape == (B, M // 2)
        assert bool(((y.double() - want).abs() <= err + 2.0 ** -24 * (want.abs() + err)).all())


@pytest.mark.parametrize("form,splits,B,M,K", [f for f in FC if f[4] < 8000])
def test_what_is_not_finite_stays_in_its_row(form, splits, B, M, K):
    g = gen(B, M, 1)
    W, _ = blocks(g, (M,), K)
    X, _ = blocks(g, (B,), K)
    assert cl.mx_fc_resolved_form(W, B) == (form, splits)
    y = cl.mx_fc_forward(W, X)
    kb = -(-K // 32)
    for n, m, at in ((0, M - 1, 0), (B - 1, 0, kb - 1), (B // 2, M // 3, kb // 2)):
        X.scales[n, at], W.scales[m, (at + kb // 3) % kb], keep = 255, 255, (int(X.scales[n, at]), int(W.scales[m, (at + kb // 3) % kb]))
        z = cl.mx_fc_forward(W, X)
        assert bool(z[n].isnan().all()) and bool(z[:, m].isnan().all())
        z[n], z[:, m] = y[n], y[:, m]
        assert torch.equal(z, y)
        X.scales[n, at], W.scales[m, (at + kb // 3) % kb] = keep


# form, tokens, experts, k, rows, K
EXPERTS = [("rows", 820, 2, 2, 42, 1426), ("rows", 1175, 4, 2, 38, 1040), ("rows", 1172, 3, 1, 50, 1029), ("rows", 1369, 3, 1, 34, 1285),
           ("tile 64", 2497, 8, 3, 34, 1482), ("tile 64", 3335, 4, 2, 34, 1053), ("tile 64", 5216, 3, 1, 50, 1210), ("tile 64", 7101, 16, 1, 34, 1378),
           ("tile 128", 4504, 16, 4, 66, 1514), ("tile 128", 6210, 40, 3, 66, 1131), ("tile 128", 11531, 40, 1, 130, 1192), ("tile 128", 11976, 16, 1, 132, 1283),
           ("tile 256 x 128", 110, 40, 4, 1484, 1423), ("tile 256 x 128", 16, 16, 3, 3858, 1026), ("tile 256 x 128", 35, 16, 1, 4340, 1200),
           ("tile 256 x 128", 35, 16, 1, 4572, 1360),
           ("tile 256", 13860, 3, 3, 130, 1443), ("tile 256", 10610, 8, 4, 136, 1032), ("tile 256", 6795, 40, 1, 914, 1415), ("tile 256", 7089, 40, 1, 966, 1292)]


def pairs_of(xv, wv, of, per):
    """The products of all pairs, float64: row n of xv is that of pairs n per .. n per + per - 1; zeros for pairs without an expert."""
    out = torch.zeros((len(of), wv.shape[1]), dtype=torch.float64, device="cuda")
    for e in range(len(wv)):
        at = (of == e).nonzero()[:, 0]
        out[at] = xv[at // per] @ wv[e].T
    return out


@pytest.mark.parametrize("form,T,E,k,M,K", EXPERTS)
def test_experts(form, T, E, k, M, K):
    g = gen(T, E, M)
    W, wv = blocks(g, (E, M), K)
    X, xv = blocks(g, (T,), K)
    chosen = torch.randint(-1, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    chosen[torch.rand((T, k), generator=g, device="cuda") < 0.01] = E + 7
    routed = ((chosen >= 0) & (chosen < E)).reshape(-1, 1).double()
    weights = torch.exp2(torch.randint(-1, 2, (T, k), generator=g, device="cuda").float())
    bias = torch.randint(-400, 401, (E, M), generator=g, device="cuda").float() / 4
    lists = cl.expert_lists(chosen, E)
    for weighted in (False, True):
        for x_per_pair in (False, True):
            assert cl.mx_experts_resolved_form(W, T, k, None, weighted, x_per_pair, True) == form
    of = chosen.reshape(-1)
    pre = pairs_of(xv, wv, of, k)
    assert torch.equal(cl.mx_experts_forward(W, X, chosen, lists=lists).double(), pre)
    with_bias = routed * (pre + bias.double()[of.clamp(0, E - 1).long()])
    relu = with_bias.clamp_min(0)
    w = weights.double().reshape(-1, 1)
    want = (w * relu).reshape(T, k, M).sum(1)
    for dtype in (torch.float32, torch.bfloat16):
        y = cl.mx_experts_forward(W, X, chosen, weights, bias, act="relu", dtype=dtype)
        assert torch.equal(y, want.to(torch.float32).to(dtype))
    # the values are their own quantisation, beside which the lists are made
    if cl.mx_experts_resolved_form(W, T, k, torch.bfloat16) == form:
        assert torch.equal(cl.mx_experts_forward(W, xv.to(torch.bfloat16), chosen, weights, bias, act="relu"), y)
    out, err = gated(with_bias / 512)
    small = cl.MxTensor(W.codes, W.scales - 9, K)
    y = cl.mx_experts_forward(small, X, chosen, None, bias / 512, act="gated", lists=lists)
    assert bool(((y.double() - out).abs() <= err + 2.0 ** -24 * (out.abs() + err)).all())
    # a row of X for each pair
    XX, xxv = blocks(g, (T * k,), K)
    pre = pairs_of(xxv, wv, of, 1)
    assert torch.equal(cl.mx_experts_forward(W, XX, chosen, x_per_pair=True, lists=lists).double(), pre)
    assert torch.equal(cl.mx_experts_forward(W, XX, chosen, weights, x_per_pair=True).double(), (w * pre).reshape(T, k, M).sum(1))


@pytest.mark.parametrize("form,T,E,k,M,K", [EXPERTS[i] for i in (0, 4, 8, 10, 13, 16, 18)])
def test_what_is_not_finite_stays_with_its_pairs(form, T, E, k, M, K):
    g = gen(T, M)
    W, _ = blocks(g, (E, M), K)
    X, _ = blocks(g, (T,), K)
    chosen = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.ones((T, k), device="cuda")
    assert cl.mx_experts_resolved_form(W, T, k) == form
    y, rows = cl.mx_experts_forward(W, X, chosen, weights), cl.mx_experts_forward(W, X, chosen)
    t, e, m, at = T // 2, E - 1, M // 2, -(-K // 32) - 1
    X.scales[t, at], W.scales[e, m, 1] = 255, 255
    z, zrows = cl.mx_experts_forward(W, X, chosen, weights), cl.mx_experts_forward(W, X, chosen)
    of_e = chosen == e
    bad = torch.zeros((T, k, M), dtype=torch.bool, device="cuda")
    bad[t] = True
    bad[:, :, m] |= of_e
    assert torch.equal(zrows.isnan(), bad.reshape(T * k, M)) and torch.equal(z.isnan(), bad.any(1))
    assert torch.equal(torch.where(zrows.isnan(), rows, zrows), rows) and torch.equal(torch.where(z.isnan(), y, z), y)


def in_a_graph_and_on_another_stream(call, inputs, eager):
    """call() writes its output; inputs are changed between replays."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = call()
    s.synchronize()
    assert torch.equal(out, eager())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(3):
        for x in inputs:
            x.copy_(torch.roll(x, 1, 0))
        out.fill_(-7.0)
        want = eager()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("form,splits,B,M,K", [("rows", 1, 17, 5755, 1033), ("tile 64", 1, 6971, 33, 1037), ("tile 64", 2, 17, 7488, 3312), ("tile 64", 8, 16, 32, 17068),
                                               ("tile 128", 8, 2049, 66, 14913), ("tile 256 x 128", 1, 9593, 398, 1348), ("tile 256", 1, 8653, 902, 1185)])
def test_workspace_graph_and_stream(form, splits, B, M, K):
    g = gen(B, M, 2)
    W, _ = blocks(g, (M,), K)
    x = blocks(g, (B,), K)[1].to(torch.bfloat16)
    assert cl.mx_fc_resolved_form(W, B, torch.bfloat16) == (form, splits)
    need = cl.mx_fc_workspace_bytes(W, B, torch.bfloat16)
    assert need >= 17 * cl.mx_row_blocks(K) * B
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    in_a_graph_and_on_another_stream(lambda: cl.mx_fc_forward(W, x, dtype=torch.float32, workspace=ws[:need]), [x], lambda: cl.mx_fc_forward(W, x, dtype=torch.float32))
    assert bool((ws[need:] == 255).all())


# joined, from one launch of the lists and from two (above 32768 pairs)
@pytest.mark.parametrize("form,T,E,k,M,K", [EXPERTS[i] for i in (0, 2, 4, 6, 12, 16, 17, 18)])
@pytest.mark.parametrize("weighted", [False, True])
def test_experts_workspace_graph_and_stream(form, T, E, k, M, K, weighted):
    g = gen(T, M, 3)
    W, _ = blocks(g, (E, M), K)
    x = blocks(g, (T,), K)[1].to(torch.bfloat16)
    chosen = torch.randint(-1, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.exp2(torch.randint(-1, 2, (T, k), generator=g, device="cuda").float()) if weighted else None
    assert cl.mx_experts_resolved_form(W, T, k, torch.bfloat16, weighted) == form
    need = binding._mx_experts_need(M, K, E, T, k, weighted, False, 0, 0, 1)
    assert need >= 17 * cl.mx_row_blocks(K) * T + 4 * T * k
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    in_a_graph_and_on_another_stream(lambda: cl.mx_experts_forward(W, x, chosen, weights, dtype=torch.float32, workspace=ws[:need]), [x, chosen],
                                     lambda: cl.mx_experts_forward(W, x, chosen, weights, dtype=torch.float32))
    assert bool((ws[need:] == 255).all())


def test_codes_beyond_32_bits():
    """One matrix, an expert's matrix and rows of X whose codes begin past 2^31 bytes, through tiles and through sixteen columns at a time."""
    K, rows = 4096, 1100003
    g = gen(7)
    few, fv = blocks(g, (1000,), K)
    codes, scales = torch.empty((rows, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((rows, K // 32), dtype=torch.uint8, device="cuda")
    for at in range(0, rows, 1000):
        n = min(1000, rows - at)
        codes[at:at + n], scales[at:at + n] = few.codes[:n], few.scales[:n]
    last = (torch.arange(rows - 1000, rows, device="cuda")) % 1000          # which of the thousand the last rows are
    far = cl.MxTensor(codes, scales, K)

    for B in (17, 1000):
        X, xv = blocks(g, (B,), K)
        assert cl.mx_fc_resolved_form(far, B) == ("tile 256 x 128", 1)
        y = cl.mx_fc_forward(far, X)
        assert torch.equal(y[:, -1000:].double(), (xv @ fv.T)[:, last])
        del y
    for M, form in ((8, "rows"), (64, "tile 128"), (200, "tile 256"), (1000, "tile 256 x 128")):
        W, wv = blocks(g, (M,), K)
        assert cl.mx_fc_resolved_form(W, rows) == (form, 1)
        assert torch.equal(cl.mx_fc_forward(W, far)[-1000:].double(), (fv @ wv.T)[last])

    E, M = 1024, 1074
    W = cl.MxTensor(codes[:E * M].view(E, M, -1), scales[:E * M].view(E, M, -1), K)
    of = torch.arange((E - 1) * M, E * M, device="cuda") % 1000
    forms = set()
    for T in (2, 80, 100000):
        X, xv = blocks(g, (T,), K)
        chosen = torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda")
        forms.add(cl.mx_experts_resolved_form(W, T, 1))
        for weights in (None, torch.full((T, 1), 0.5, device="cuda")):
            y = cl.mx_experts_forward(W, X, chosen, weights)
            assert torch.equal(y.double(), (xv @ fv.T)[:, of] * (1.0 if weights is None else 0.5))
    assert forms == {"rows", "tile 64", "tile 128"}
