"""Every form of the 8-bit products, named, and what is about how they run: workspaces, streams, recorded calls, guarded memory, values that are not finite, offsets beyond 32 bits.
References are fp64 products on the GPU, with the gates of f8_ref."""
import numpy as np
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu
F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, ref.F8


def wide(q):
    """What an F8Tensor stands for, float64 on its device; of a gated matrix each half with its own scales."""
    v = q.values.double()
    if q.gated:
        (a, b), (s, t) = v.chunk(2), q.scales.double().chunk(2)
        parts = [(a, s), (b, t)]
    else:
        parts = [(v, q.scales.double())]
    kb = cl.f8_row_blocks(q.K)
    return torch.cat([p * s[:, :kb].repeat_interleave(q.block_rows, 0)[:len(p)].repeat_interleave(128, 1) for p, s in parts])[:, :q.K]


def eights(x, w):
    K = x.shape[1]
    x, w = (torch.nn.functional.pad(v.abs(), (0, -K % 8)).float() for v in (x, w))
    total = torch.zeros((len(x), len(w)), device=x.device)
    for k in range(0, x.shape[1], 8):
        most = x[:, k, None] * w[:, k]
        for i in range(1, 8):
            torch.maximum(most, x[:, k + i, None] * w[:, k + i], out=most)
        total += most
    return total.double() * (1 + K * 2.0 ** -23)


def product(x, w, bias, act, narrow):
    """-> (result, bound), as f8_ref.product."""
    pre, size = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        pre, size = pre + bias.double(), size + bias.double().abs()
    err = (x.shape[1] + 8) * 2.0 ** -23 * size
    if narrow:
        err = err + 7 * 2.0 ** -13 * eights(x, w)
    if act == "gated":
        (g, u), (eg, eu) = pre.chunk(2, 1), err.chunk(2, 1)
        silu = g * torch.sigmoid(g)
        out = silu * u
        return out, 1.1 * u.abs() * eg + (silu.abs() + 1.1 * eg) * eu + out.abs() * (8 + g.abs()) * 2.0 ** -23
    return (pre.clamp_min(0) if act == "relu" else pre), err


def check(y, want, err, what):
    if isinstance(y, cl.F8Tensor):
        ref.assert_f8_within(y, want.cpu().numpy(), err.cpu().numpy(), what)
        return
    bound = err + ref.mx_ref.HALF_ULP[y.dtype] * (want.abs() + err) + ref.mx_ref.SMALLEST[y.dtype]
    off = (y.double() - want).abs()
    if y.dtype == F16:                                       # (what fp16 rounds to Inf: 65520 and more)
        off = torch.where(y.isinf() & (y.sign() == want.sign()) & (want.abs() + err >= 65520), torch.zeros_like(off), off)
    assert bool((off <= bound).all()), (what, float((off / bound).max()), int((off > bound).sum()))


def same(a, b):
    if isinstance(a, cl.F8Tensor):
        return torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)
    return torch.equal(a, b)


def draw(B, M, K, gated, seed, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(rows):
        return cl.f8_quantize(torch.randn((rows, K), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda")) * K ** -0.5, 128)

    W = cl.f8_gated(matrix(M), matrix(M)) if gated else matrix(M)
    X = (torch.randn((B, K), generator=g, device="cuda") * torch.exp(torch.randn((B, 1), generator=g, device="cuda"))).to(dtype)
    return W, X, 0.3 * torch.randn(len(W.values), generator=g, device="cuda")


# form, splits, batch, outputs, K, type of X, of the output, activation
FORMS = [
    ("few numbers", 1, 1, 23, 34, BF16, BF16, "gated"), ("few numbers", 1, 16, 1000, 4096, F32, F32, "relu"), ("few numbers", 1, 5, 333, 1700, F16, F8, "gated"),
    ("few numbers", 1, 7, 129, 515, BF16, F8, "none"), ("few", 1, 9, 5614, 5596, F16, F8, "gated"), ("few", 1, 29, 38, 4639, BF16, BF16, "none"), ("few", 1, 31, 23, 5068, F32, F32, "gated"),
    ("few", 1, 20, 30, 4358, F16, F8, "none"),
    ("tile 64", 1, 426, 25, 42, BF16, BF16, "gated"), ("tile 64", 1, 343, 18, 69, BF16, BF16, "none"), ("tile 64", 1, 335, 18, 49, F16, F8, "gated"), ("tile 64", 1, 367, 19, 69, F8, F32, "gated"),
    ("tile 64", 2, 284, 31, 722, F16, F8, "gated"), ("tile 64", 4, 351, 17, 3200, BF16, BF16, "relu"), ("tile 64", 8, 3, 32, 24400, F16, F8, "none"), ("tile 64", 8, 6, 17, 15527, F32, F32, "gated"),
    ("tile 128", 1, 169, 6980, 33, F8, BF16, "gated"), ("tile 128", 1, 258, 7158, 36, BF16, BF16, "none"), ("tile 128", 1, 381, 19, 81, F16, F8, "none"), ("tile 128", 1, 300, 500, 100, F8, F8, "none"),
    ("tile 128", 1, 150, 6948, 1798, F8, F8, "gated"), ("tile 128", 1, 8118, 220, 34, F32, F32, "none"), ("tile 128", 2, 70, 6741, 2513, F16, F8, "gated"), ("tile 128", 4, 66, 6995, 1963, F16, F8, "none"),
    ("tile 128", 8, 71, 3268, 6900, F32, F32, "relu"), ("tile 128", 8, 104, 1555, 10491, F8, F32, "gated"),
    # (more tiles than compute units: workgroups go from one to the next, with one step to a tile, with three, and with more than fours of them)
    ("tile 256", 1, 1258, 223, 33, F8, F8, "gated"), ("tile 256", 1, 5644, 2196, 38, F8, F8, "none"), ("tile 256", 1, 5537, 1166, 35, BF16, BF16, "gated"), ("tile 256", 1, 4300, 2200, 260, F8, F8, "gated"),
    ("tile 256", 1, 5000, 2500, 130, BF16, F8, "none"), ("tile 256", 1, 5100, 2470, 900, BF16, BF16, "none"), ("tile 256", 4, 3485, 141, 14150, F8, F8, "gated"), ("tile 256", 8, 4704, 131, 24334, BF16, BF16, "none"),
    # (outputs in fp32, or in 8 bits of an input in fp16: 256 x 128)
    ("tile 256", 1, 6024, 359, 36, F32, F32, "gated"), ("tile 256", 1, 9000, 1500, 300, F32, F32, "relu"), ("tile 256", 8, 129, 3911, 18938, F32, F32, "none"), ("tile 256", 2, 2657, 530, 10655, F16, F8, "gated"),
]


@pytest.mark.parametrize("form,splits,B,M,K,x_type,y_type,act", FORMS)
def test_form(form, splits, B, M, K, x_type, y_type, act):
    W, X, bias = draw(B, M, K, act == "gated", B + M + K, BF16 if x_type == F8 else x_type)
    if x_type == F8:
        X = cl.f8_quantize(X)
    assert cl.f8_fc_resolved_form(W, B, x_type, act, y_type) == (form, splits)
    x = wide(X if x_type == F8 else cl.f8_quantize(X))
    narrow = y_type in (BF16, F16)
    for b in (None, bias):
        want, err = product(x, wide(W), b, act, narrow)
        y = cl.f8_fc_forward(W, X, b, act=act, dtype=y_type)
        check(y, want, err, (form, b is None))
        assert same(y, cl.f8_fc_forward(W, X, b, act=act, dtype=y_type))                 # run to run


@pytest.mark.parametrize("act", ["none", "gated"])
@pytest.mark.parametrize("x_type,y_type", [(F32, F32), (BF16, BF16), (BF16, F8), (F16, F8), (F8, F16)])
@pytest.mark.parametrize("M,K,largest,batches", [(2048, 9216, 256, (1, 32, 64, 128, 192, 255, 256)), (962, 7400, 700, (5, 33, 100, 265, 500)), (640, 300, 4096, (1, 40, 300, 1000, 4000))])
def test_the_workspace_of_the_largest_batch_serves_all(M, K, largest, batches, x_type, y_type, act):
    W, X, _ = draw(largest, M, K, act == "gated", M, BF16 if x_type == F8 else x_type)
    need = cl.f8_fc_workspace_bytes(W, largest, x_type, act, y_type)
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    w = wide(W)
    for batch in batches:
        part = X[:batch]
        q = cl.f8_quantize(part)
        want, err = product(wide(q), w, None, act, y_type in (BF16, F16))
        y = cl.f8_fc_forward(W, q if x_type == F8 else part, act=act, dtype=y_type, workspace=room[:need])
        check(y, want, err, batch)
        assert bool((room[need:] == 255).all())


def test_what_is_beside_the_output_stays():
    for B, M, K, act, dtype in ((3, 100, 300, "none", BF16), (70, 131, 700, "gated", F16), (300, 257, 200, "none", F32), (2034, 90, 33, "gated", BF16), (1100, 1000, 256, "none", BF16)):
        W, X, _ = draw(B, M, K, act == "gated", B, dtype)
        room = torch.full((B + 2, M), 7.0, dtype=dtype, device="cuda")
        y = cl.f8_fc_forward(W, X, act=act, out=room[1:B + 1])
        assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all()) and torch.equal(y, cl.f8_fc_forward(W, X, act=act))
        # 8-bit outputs: rows of values and of scales
        kb, pitch = cl.f8_row_blocks(M), cl.f8_row_scales(M)
        values, scales = torch.full((B + 2, kb * 128), 1.0, device="cuda").to(F8), torch.full((B + 2, pitch), 7.0, device="cuda")
        out = cl.F8Tensor(values[1:B + 1], scales[1:B + 1], M)
        cl.f8_fc_forward(W, X, act=act, out=out)
        assert bool((values[0].float() == 1).all()) and bool((values[-1].float() == 1).all()) and bool((scales[0] == 7).all()) and bool((scales[-1] == 7).all())
        assert same(out, cl.f8_fc_forward(W, X, act=act, dtype=F8)) and bool((out.values[:, M:].float() == 0).all()) and bool((out.scales[:, kb:] == 0).all())
        cl.rms_norm(y, out=out, dtype=F8)
        assert bool((values[0].float() == 1).all()) and bool((values[-1].float() == 1).all()) and bool((scales[0] == 7).all()) and bool((scales[-1] == 7).all())


def test_rows_at_odd_addresses():
    for dtype in ref.DTYPES:
        for B, K in ((3, 517), (40, 200), (600, 333)):
            W, X, _ = draw(B, 300, K, False, B, dtype)
            pitch = K + 3
            buf = torch.full((B * pitch + 1,), float("nan"), dtype=dtype, device="cuda")
            odd = buf[1:].view(B, pitch)[:, :K]
            odd.copy_(X)
            assert torch.equal(cl.f8_fc_forward(W, odd), cl.f8_fc_forward(W, X))


@pytest.mark.parametrize("B,M,K,act,y_type", [(4, 300, 700, "none", BF16), (70, 300, 700, "gated", BF16), (300, 500, 100, "none", BF16), (300, 500, 400, "none", F8), (5000, 2500, 130, "none", BF16),
                                              (4300, 2200, 260, "gated", F8), (5537, 1166, 35, "gated", BF16)])
def test_what_is_not_finite_stays_in_its_row(B, M, K, act, y_type):
    W, X, _ = draw(B, M, K, act == "gated", B)
    before = cl.f8_fc_forward(W, X, act=act, dtype=y_type)
    bad = torch.zeros(B, dtype=torch.bool, device="cuda")
    bad[torch.arange(0, B, 3, device="cuda")] = True
    X[bad, K // 2] = float("nan")
    X[0, 0], X[0, K // 2] = float("inf"), 1.0
    y = cl.f8_fc_forward(W, X, act=act, dtype=y_type)
    if y_type == F8:
        assert bool(y.scales[bad, :cl.f8_row_blocks(M)].isnan().all()) and torch.equal(y.values.view(torch.uint8)[~bad], before.values.view(torch.uint8)[~bad]) and torch.equal(y.scales[~bad], before.scales[~bad])
    else:
        assert bool(y[bad].isnan().all()) and torch.equal(y[~bad], before[~bad])
    # ... and of a block of W in the outputs of its 128 rows
    W.scales[0, 0] = float("nan")
    X[bad] = 1.0
    y = cl.f8_fc_forward(W, X, act=act, dtype=BF16)
    n = min(128, M)
    assert bool(y[:, :n].isnan().all()) and not bool(y[:, n:].isnan().any())


def test_another_stream():
    W, X, _ = draw(300, 1000, 2050, True, 3)
    want = cl.f8_fc_forward(W, X, act="gated", dtype=F8)
    n, total = cl.rms_norm(X, residual=X, dtype=F8)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = torch.zeros_like(X)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(X)
        y = cl.f8_fc_forward(W, late, act="gated", dtype=F8)
        m, t = cl.rms_norm(late, residual=late, dtype=F8)
    side.synchronize()
    assert same(y, want) and same(m, n) and torch.equal(t, total)


@pytest.mark.parametrize("B,M,K,act,y_type", [(1, 500, 900, "none", BF16), (20, 300, 700, "gated", F8), (64, 1000, 9216, "none", F32), (300, 500, 400, "none", F8), (5000, 2500, 130, "none", BF16)])
def test_recorded(B, M, K, act, y_type):
    W, X, bias = draw(B, M, K, act == "gated", B, F32 if y_type == F32 else BF16)
    run = lambda: (cl.f8_fc_forward(W, X, bias, act=act, dtype=y_type), cl.f8_quantize(X), cl.rms_norm(X, residual=X, dtype=F8)[0])  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in range(4):
        X.copy_(draw(B, M, K, False, seed + 50)[1])
        graph.replay()
        kept = [(g.values.clone(), g.scales.clone()) if isinstance(g, cl.F8Tensor) else g.clone() for g in got]
        torch.cuda.synchronize()
        for a, b in zip(kept, run()):
            assert torch.equal(a, b) if not isinstance(b, cl.F8Tensor) else (torch.equal(a[0].view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a[1], b.scales)), seed


def test_offsets_beyond_32_bits():
    # outputs, then inputs, of more than 2^32 bytes: a few rows of each end against a product of those alone
    for B, M, K in ((70000, 33000, 128), (70000, 128, 66000)):
        g = torch.Generator(device="cuda").manual_seed(M)
        W = cl.f8_quantize(torch.randn((M, K), generator=g, device="cuda") * K ** -0.5, 128)
        X = torch.randn((B, K), generator=g, device="cuda", dtype=BF16)
        y = cl.f8_fc_forward(W, X)
        for rows in (slice(0, 300), slice(B // 2, B // 2 + 300), slice(B - 300, B)):
            part = X[rows].contiguous()
            check(y[rows], *product(wide(cl.f8_quantize(part)), wide(W), None, "none", True), rows)
        del y
        n = cl.rms_norm(X, dtype=F8)
        q = cl.f8_quantize(X)
        for rows in (slice(0, 5), slice(B - 5, B)):
            assert same(cl.F8Tensor(n.values[rows], n.scales[rows], K), cl.rms_norm(X[rows], dtype=F8)) and same(cl.F8Tensor(q.values[rows], q.scales[rows], K), cl.f8_quantize(X[rows]))
            assert torch.equal(cl.f8_dequantize(q, BF16)[rows], cl.f8_dequantize(cl.F8Tensor(q.values[rows], q.scales[rows], K), BF16))
        del X, n, q
    # one row of the most elements
    X = torch.randn((1, 1 << 24), generator=g, device="cuda")
    W = cl.f8_quantize(torch.randn((16, 1 << 24), generator=g, device="cuda") * 2.0 ** -12, 128)
    x, w = wide(cl.f8_quantize(X)), wide(W)
    size = x.abs() @ w.abs().T
    assert bool(((cl.f8_fc_forward(W, X).double() - x @ w.T).abs() <= ((1 << 24) // 128 + 136) * 2.0 ** -23 * size).all())


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("rows,K", [(70000, 100), (40000, 257), (9000, 4100), (3000, 20000), (20000, 1024)])
def test_norm_of_many_rows(rows, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(K)
    x, r = (torch.randn((rows, K), generator=g, device="cuda").to(dtype) for _ in range(2))
    gain = torch.randn(K, generator=g, device="cuda")
    for residual in (None, r):
        y = cl.rms_norm(x, gain, 1e-5, residual=residual, dtype=F32)
        q = cl.rms_norm(x, gain, 1e-5, residual=residual, dtype=F8)
        h = x
        if residual is not None:
            (y, total), (q, again) = y, q
            h = (x.float() + r.float()).to(dtype)
            assert torch.equal(total, h) and torch.equal(again, h)
        h = h.double()
        want = h / (h.square().mean(1, keepdim=True) + 1e-5).sqrt() * gain.double()
        off = (y.double() - want).abs()
        assert bool((off <= want.abs() * (0.5 * (64 + 8 + K / 1024 + 22 + 2) + 6) * 2.0 ** -24).all())
        assert same(q, cl.f8_quantize(y))


def test_other_devices_and_shapes_are_refused():
    W, X, bias = draw(4, 256, 300, False, 1)
    q = cl.f8_quantize(X)
    rows = cl.f8_quantize(torch.randn((256, 300), device="cuda"))
    gated = cl.f8_gated(cl.f8_quantize(torch.randn((100, 300), device="cuda"), 128), cl.f8_quantize(torch.randn((100, 300), device="cuda"), 128))
    for call in (lambda: cl.f8_fc_forward(rows, X), lambda: cl.f8_fc_forward(W, X[:, :200]), lambda: cl.f8_fc_forward(W, X.cpu()), lambda: cl.f8_fc_forward(W, X.double()), lambda: cl.f8_fc_forward(W, X, bias[:5]),
                 lambda: cl.f8_fc_forward(W, X, act="other"), lambda: cl.f8_fc_forward(gated, X), lambda: cl.f8_fc_forward(W, W), lambda: cl.f8_fc_forward(W, X, out=torch.empty((4, 255), device="cuda")),
                 lambda: cl.f8_fc_forward(W, X, out=q), lambda: cl.f8_fc_forward(W, X.t().contiguous().t()), lambda: cl.f8_quantize(X[0]), lambda: cl.f8_quantize(X, out=rows),
                 lambda: cl.f8_dequantize(gated), lambda: cl.f8_gated(W, rows), lambda: cl.F8Tensor(q.values, q.scales, 500), lambda: cl.F8Tensor(q.values.view(torch.uint8), q.scales, 300),
                 lambda: cl.F8Tensor(W.values, W.scales, 300), lambda: cl.rms_norm(X, residual=X.float()), lambda: cl.rms_norm(X, torch.ones(299, device="cuda")), lambda: cl.rms_norm(X, torch.ones(300, device="cuda", dtype=F16)),
                 lambda: cl.rms_norm(X, sum_out=X), lambda: cl.rms_norm(X, residual=X, sum_out=X[:2]), lambda: cl.rms_norm(X, out=q, dtype=BF16), lambda: cl.rms_norm(X, out=torch.empty((4, 300), device="cuda"), dtype=BF16),
                 lambda: cl.rms_norm(X.cpu()), lambda: cl.rms_norm(X, torch.ones(300))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: cl.f8_quantize(X, 64), lambda: cl.rms_norm(X, eps=-1.0), lambda: cl.rms_norm(X, residual=X, sum_out=X, out=X), lambda: cl.f8_fc_forward(W, torch.empty((600, 300), device="cuda"), workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(cl.CLError):
            call()
