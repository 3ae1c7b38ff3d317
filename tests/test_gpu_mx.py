"""Microscaled 4-bit quantisation, back, and the product, against their plain fp64 forms (mx_ref)."""
import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


def same_blocks(q, x):
    codes, scales = ref.quantise(x.double().cpu().numpy())
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)


def spread(rng, shape, dtype):
    """Values over many binades, zeros, and exact ties of the grid among them."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-6, 7, shape)
    x = np.where(rng.random(shape) < 0.2, rng.integers(-24, 25, shape) / 4.0, x)
    x = np.where(rng.random(shape) < 0.1, 0.0, x)
    return torch.from_numpy(x).to("cuda", dtype)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 31), (3, 32), (5, 33), (2, 127), (7, 129), (4, 4100), (65, 1000), (300, 96)])
def test_quantise_and_back(rows, K, dtype):
    x = spread(np.random.default_rng(rows * K), (rows, K), dtype)
    q = cl.mx_quantize(x)
    assert q.shape == (rows, K)
    same_blocks(q, x)
    for out in ref.DTYPES:
        want = torch.from_numpy(ref.values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), K)).to(out)
        assert torch.equal(cl.mx_dequantize(q, out).cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_16_bit_value(dtype):
    """Each value once as the largest of a block and once beside every other exponent: a row of all bit patterns in order, and shuffled."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    rng = np.random.default_rng(1)
    x = torch.stack([every, every[torch.from_numpy(rng.permutation(65536))], torch.where(every.isfinite(), every, torch.zeros_like(every))]).cuda()
    same_blocks(cl.mx_quantize(x), x)


def test_extreme_fp32_values():
    big, tiny, least = 3.4028234663852886e38, 2.0 ** -126, 2.0 ** -149
    vals = [big, -big, tiny, -tiny, least, tiny * 0.75, 2.0 ** -127, 2.0 ** -125, 2.0 ** -124, 7.999999, 6.0, 5.0, 4.999999, 5.000001, 0.25, 0.2500001, 0.0, -0.0]
    x = torch.zeros((len(vals) + 3, 64))
    for i, v in enumerate(vals):
        x[i, 3], x[i, 40], x[i, 41] = v, v, v / 4
    x[-3, 5], x[-2, 5], x[-1, 5] = float("nan"), float("inf"), -float("inf")
    x[-3:, 6], x[-3:, 40] = 1.0, 2.0
    x = x.cuda()
    q = cl.mx_quantize(x)
    same_blocks(q, x)
    v = cl.mx_dequantize(q)
    assert v[-3:, :32].isnan().all() and v[-3:, 32:].isfinite().all() and (v[-3:, 40] == 2).all()


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("first,stride", [(0, 200), (1, 200), (3, 203), (8, 208)])
def test_rows_at_a_distance(dtype, first, stride):
    rng = np.random.default_rng(stride)
    buf = spread(rng, (9, stride), dtype)
    x = buf.view(-1)[first:first + 8 * stride].view(8, stride)[:, :150]
    q = cl.mx_quantize(x)
    same_blocks(q, x)
    out = torch.full((8, stride), 7.0, dtype=dtype, device="cuda")
    cl.mx_dequantize(q, out=out[:, :150])
    assert torch.equal(out[:, :150], cl.mx_dequantize(q, dtype)) and bool((out[:, 150:] == 7).all())


def test_no_rows():
    q = cl.mx_quantize(torch.empty((0, 70), device="cuda"))
    assert q.shape == (0, 70) and cl.mx_dequantize(q).shape == (0, 70)
    W = cl.mx_quantize(torch.ones((5, 70), device="cuda"))
    assert cl.mx_fc_forward(W, torch.empty((0, 70), device="cuda")).shape == (0, 5)


def test_a_stack_of_matrices():
    x = spread(np.random.default_rng(5), (3, 10, 77), torch.float32)
    q = cl.mx_quantize(x)
    assert q.shape == (3, 10, 77)
    for i in range(3):
        codes, scales = ref.quantise(x[i].double().cpu().numpy())
        assert np.array_equal(q.codes[i].cpu().numpy(), codes) and np.array_equal(q.scales[i].cpu().numpy(), scales)
    assert torch.equal(cl.mx_dequantize(q)[1], cl.mx_dequantize(cl.mx_quantize(x[1])))


# batch, rows, K
SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 31), (3, 100, 513), (15, 33, 127), (16, 64, 512), (17, 130, 640), (33, 48, 1000), (64, 128, 256), (65, 96, 4100),
          (130, 259, 384), (1, 4096, 1030), (8, 1000, 4096), (300, 257, 2050), (513, 300, 700), (5, 20, 9000)]


def operands(rng, B, M, K, dtype):
    x = spread(rng, (B, K), dtype)
    w = cl.mx_quantize(torch.from_numpy((rng.standard_normal((M, K)) * 0.02).astype(np.float32)).cuda())
    wq = ref.values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), K)
    return x, w, ref.quantised(x.double().cpu().numpy()), wq


@pytest.mark.parametrize("B,M,K", SHAPES)
def test_product(B, M, K):
    rng = np.random.default_rng(B + M + K)
    for i, dtype in enumerate(ref.DTYPES):
        x, w, xq, wq = operands(rng, B, M, K, dtype)
        bias = rng.standard_normal(M).astype(np.float32) if i != 1 else None
        relu = i == 0
        bd = None if bias is None else torch.from_numpy(bias).cuda()
        y = cl.mx_fc_forward(w, x, bd, relu=relu)
        assert y.dtype == dtype
        want, err = ref.product(xq, wq, bias, "relu" if relu else "none")
        ref.assert_within(y, want, err, (B, M, K, dtype))
        assert torch.equal(y, cl.mx_fc_forward(w, x, bd, relu=relu))                      # run to run
        # quantised beforehand, and other output types
        q = cl.mx_quantize(x)
        for out in ref.DTYPES:
            z = cl.mx_fc_forward(w, q, bd, relu=relu, dtype=out)
            ref.assert_within(z, want, err, (B, M, K, dtype, out))
            if out == dtype:
                assert torch.equal(z, y)


@pytest.mark.parametrize("B,M,K", [(1, 2, 40), (4, 66, 300), (40, 130, 512), (200, 514, 300)])
def test_gated_product(B, M, K):
    rng = np.random.default_rng(B * M)
    x, w, xq, wq = operands(rng, B, M, K, torch.float32)
    bias = rng.standard_normal(M).astype(np.float32)
    for b in (None, bias):
        y = cl.mx_fc_forward(w, x, None if b is None else torch.from_numpy(b).cuda(), act="gated")
        assert y.shape == (B, M // 2)
        ref.assert_within(y, *ref.product(xq, wq, b, "gated"), (B, M, K))


@pytest.mark.parametrize("B,M,K", [(3, 40, 300), (40, 70, 1000), (300, 300, 1100)])
def test_what_is_not_finite_stays_in_its_row(B, M, K):
    rng = np.random.default_rng(B)
    x, w, _, _ = operands(rng, B, M, K, torch.float32)
    y = cl.mx_fc_forward(w, x)
    x2 = x.clone()
    x2[B // 2, K // 2] = float("inf")
    y2 = cl.mx_fc_forward(w, x2)
    rest = torch.arange(B, device="cuda") != B // 2
    assert y2[B // 2].isnan().all() and torch.equal(y2[rest], y[rest])
    w.scales[M // 3, 0] = 255
    y3 = cl.mx_fc_forward(w, x, relu=True)
    rest = torch.arange(M, device="cuda") != M // 3
    assert y3[:, M // 3].isnan().all() and torch.equal(y3[:, rest], torch.relu(y[:, rest]))


@pytest.mark.parametrize("B", [2, 70, 300])
def test_product_of_rows_at_a_distance_into_given_memory(B):
    rng = np.random.default_rng(B)
    M, K = 75, 333
    buf = spread(rng, (B, 401), torch.bfloat16)
    x = buf[:, 5:5 + K]
    _, w, _, wq = operands(rng, 1, M, K, torch.float32)
    out = torch.full((B, M), 9.0, device="cuda")
    ws = torch.full((cl.mx_fc_workspace_bytes(w, B, torch.bfloat16) + 256,), 255, dtype=torch.uint8, device="cuda")
    y = cl.mx_fc_forward(w, x, dtype=torch.float32, out=out, workspace=ws)
    assert y.data_ptr() == out.data_ptr()
    ref.assert_within(y, *ref.product(ref.quantised(x.double().cpu().numpy()), wq, None, "none"))
    assert bool((ws[-256:] == 255).all())


@pytest.mark.parametrize("B", [1, 20, 400])
def test_captured_and_on_another_stream(B):
    rng = np.random.default_rng(B)
    x, w, xq, wq = operands(rng, B, 200, 600, torch.float32)
    want, err = ref.product(xq, wq, None, "none")
    out = torch.zeros((B, 200), device="cuda")
    ws = torch.empty(cl.mx_fc_workspace_bytes(w, B, torch.float32), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cl.mx_fc_forward(w, x, out=out, workspace=ws)
    s.synchronize()
    ref.assert_within(out, want, err)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cl.mx_fc_forward(w, x, out=out, workspace=ws)
    for i in range(3):
        x.copy_(x * (i + 1))
        out.zero_()
        eager = cl.mx_fc_forward(w, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_refusals_of_the_binding():
    x = torch.ones((4, 64), device="cuda")
    q = cl.mx_quantize(x)
    for bad in (x.double(), x.t(), x[0], x.cpu()):
        with pytest.raises(ValueError):
            cl.mx_fc_forward(q, bad)
    with pytest.raises(ValueError):
        cl.mx_quantize(x, out=cl.mx_quantize(torch.ones((4, 65), device="cuda")))
    with pytest.raises(ValueError):
        cl.mx_quantize(x.long())
    with pytest.raises(ValueError):
        cl.MxTensor(q.codes, q.scales, 129)
    with pytest.raises(ValueError):
        cl.MxTensor(q.codes.float(), q.scales, 64)
    with pytest.raises(ValueError):
        cl.mx_fc_forward(q, x, bias=torch.ones(5, device="cuda"))
    with pytest.raises(ValueError):
        cl.mx_fc_forward(q, x, act="tanh")
    with pytest.raises(ValueError):
        cl.mx_fc_forward(q, x, out=torch.ones((4, 5), device="cuda"))
    with pytest.raises(cl.CLError):
        cl.mx_fc_forward(cl.mx_quantize(torch.ones((3, 64), device="cuda")), x, act="gated")
    with pytest.raises(cl.CLError):
        cl.mx_fc_forward(q, torch.ones(((1 << 20) + 16, 64), device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
