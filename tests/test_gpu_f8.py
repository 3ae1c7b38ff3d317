"""Quantisation to 8 bits with a scale for each block of 128, back, the norm that hands its output on in 8 bits, and the products, against their plain forms (f8_ref)."""
import numpy as np
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


def same_blocks(q, x, block_rows=1):
    v, s = ref.quantise(x.float().cpu().numpy(), block_rows)
    got, scales = ref.stored(q)
    kb = s.shape[1]
    assert np.array_equal(scales[:, :kb], s, equal_nan=True) and (scales[:, kb:] == 0).all()
    assert np.array_equal(got, v) and np.array_equal(np.signbit(got), np.signbit(v))


def spread(rng, shape, dtype):
    """Values over many binades, zeros of both signs, and multiples of an eighth among them."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-8, 9, shape)
    x = np.where(rng.random(shape) < 0.2, rng.integers(-64, 65, shape) / 8.0, x)
    x = np.where(rng.random(shape) < 0.1, np.where(rng.random(shape) < 0.5, 0.0, -0.0), x)
    return torch.from_numpy(x).to("cuda", dtype)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 127), (3, 128), (5, 129), (127, 130), (128, 512), (129, 513), (4, 4100), (65, 1000), (300, 96)])
def test_quantise_and_back(rows, K, dtype, block_rows):
    x = spread(np.random.default_rng(rows * K), (rows, K), dtype)
    q = cl.f8_quantize(x, block_rows)
    assert q.shape == (rows, K) and q.block_rows == block_rows
    same_blocks(q, x, block_rows)
    for out in ref.DTYPES:
        want = torch.from_numpy(ref.stand_for(q)).float().to(out)        # (the product in fp32, then the type)
        assert torch.equal(cl.f8_dequantize(q, out).cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_16_bit_value(dtype):
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    rng = np.random.default_rng(1)
    x = torch.stack([every, every[torch.from_numpy(rng.permutation(65536))], torch.where(every.isfinite(), every, torch.zeros_like(every))]).cuda()
    same_blocks(cl.f8_quantize(x), x)


def test_extreme_fp32_values():
    big, tiny, least = 3.4028234663852886e38, 2.0 ** -126, 2.0 ** -149
    vals = [big, -big, tiny, -tiny, least, tiny * 448, float(np.nextafter(np.float32(tiny * 448), np.float32(0))), 448.0, 464.0, 2.0 ** -117, 1e-40, 0.0, -0.0]
    x = torch.zeros((len(vals) + 3, 256))
    for i, v in enumerate(vals):
        x[i, 3], x[i, 140], x[i, 141], x[i, 142] = v, v, v / 4, v * 0.2
    x[-3, 5], x[-2, 5], x[-1, 5] = float("nan"), float("inf"), -float("inf")
    x[-3:, 6], x[-3:, 140] = 1.0, 2.0
    x = x.cuda()
    q = cl.f8_quantize(x)
    same_blocks(q, x)
    v = cl.f8_dequantize(q)
    assert v[-3:, :128].isnan().all() and v[-3:, 128:].isfinite().all() and (v[-3:, 140] == 2).all()
    w = torch.zeros((300, 256), device="cuda")
    w[:len(x)], w[200, 200] = x, float("inf")
    same_blocks(cl.f8_quantize(w, 128), w, 128)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("first,stride", [(0, 200), (1, 200), (3, 203), (8, 208)])
def test_rows_at_a_distance(dtype, first, stride, block_rows):
    rng = np.random.default_rng(stride)
    buf = spread(rng, (9, stride), dtype)
    x = buf.view(-1)[first:first + 8 * stride].view(8, stride)[:, :150]
    q = cl.f8_quantize(x, block_rows)
    same_blocks(q, x, block_rows)
    out = torch.full((8, stride), 7.0, dtype=dtype, device="cuda")
    cl.f8_dequantize(q, out=out[:, :150])
    assert torch.equal(out[:, :150], cl.f8_dequantize(q, dtype)) and bool((out[:, 150:] == 7).all())


def test_a_stack_of_rows_and_no_rows():
    x = spread(np.random.default_rng(5), (3, 10, 77), torch.float32)
    q = cl.f8_quantize(x)
    assert q.shape == (3, 10, 77) and torch.equal(cl.f8_dequantize(q)[1], cl.f8_dequantize(cl.f8_quantize(x[1])))
    q = cl.f8_quantize(torch.empty((0, 70), device="cuda"))
    assert q.shape == (0, 70) and cl.f8_dequantize(q).shape == (0, 70)
    W = cl.f8_quantize(torch.ones((5, 70), device="cuda"), 128)
    assert cl.f8_fc_forward(W, torch.empty((0, 70), device="cuda")).shape == (0, 5)
    assert cl.rms_norm(torch.empty((0, 70), device="cuda"), dtype=ref.F8).shape == (0, 70)


# --------------------------------------------------------------------------- #
# the norm
# --------------------------------------------------------------------------- #
def normed(x, gain, eps, residual):
    """-> (h as float64, result, bound)"""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h = h.double().cpu().numpy()
    return (h,) + ref.norm(h, None if gain is None else gain.double().cpu().numpy(), eps)


NORMS = [(1, 1), (1, 8), (7, 31), (5, 127), (300, 128), (33, 129), (9, 520), (4, 1000), (3, 4096), (3, 4100), (2, 8200), (5, 16384), (2, 33000), (2, 65537), (1, 140000)]


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("rows,K", NORMS)
def test_norm(rows, K, dtype):
    rng = np.random.default_rng(rows + K)
    x, r = spread(rng, (rows, K), dtype), spread(rng, (rows, K), dtype)
    for n, (gain, residual, eps) in enumerate([(None, None, 1e-6), (torch.float32, r, 1e-5), (dtype, r, 0.0), (dtype, None, 1e-3)]):
        g = None if gain is None else torch.from_numpy(1 + 0.3 * rng.standard_normal(K)).to("cuda", gain)
        keep = x.clone(), r.clone()
        h, want, err = normed(x, g, eps, residual)
        if eps == 0:
            want, err = np.where((h == 0).all(1, keepdims=True), np.nan, want), err
        for out in ref.DTYPES + [ref.F8]:
            y = cl.rms_norm(x, g, eps, residual=residual, dtype=out)
            if residual is not None:
                y, total = y
                assert total.dtype == dtype and np.array_equal(total.double().cpu().numpy(), h)
            if out == ref.F8:
                q = cl.f8_quantize(cl.rms_norm(x, g, eps, residual=residual, dtype=torch.float32)[0] if residual is not None else cl.rms_norm(x, g, eps, dtype=torch.float32))
                assert torch.equal(y.values.view(torch.uint8), q.values.view(torch.uint8)) and np.array_equal(y.scales.cpu(), q.scales.cpu(), equal_nan=True)
                ref.assert_f8_within(y, want, err, (rows, K, dtype, n))
            else:
                ref.assert_within(y, want, err, (rows, K, dtype, out, n))
        assert torch.equal(x, keep[0]) and torch.equal(r, keep[1])


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("K", [100, 4100, 70000])
def test_norm_in_place_and_at_a_distance(dtype, K):
    rng = np.random.default_rng(K)
    pitch = K + 13
    buf = spread(rng, (6, pitch), dtype)
    x, r = buf.view(-1)[1:1 + 5 * pitch].view(5, pitch)[:, :K], spread(rng, (5, K + 2), dtype)[:, :K]
    g = torch.from_numpy(rng.standard_normal(K)).to("cuda", dtype)
    want, total = cl.rms_norm(x.contiguous(), g, residual=r.contiguous())
    # the sum in the residual's place, the output in X's
    x2, r2 = torch.full((5, pitch), 9.0, dtype=dtype, device="cuda"), r.clone()
    x2[:, :K] = x
    y, t = cl.rms_norm(x2[:, :K], g, residual=r2, out=x2[:, :K], sum_out=r2)
    assert y.data_ptr() == x2.data_ptr() and t is r2 and torch.equal(y, want) and torch.equal(r2, total) and bool((x2[:, K:] == 9).all())
    # the sum in X's place
    x3 = x.clone()
    y, t = cl.rms_norm(x3, g, residual=r, sum_out=x3)
    assert torch.equal(y, want) and torch.equal(x3, total)
    y, t = cl.rms_norm(x, g, residual=r, dtype=ref.F8)
    q, _ = cl.rms_norm(x.contiguous(), g, residual=r.contiguous(), dtype=ref.F8)
    assert torch.equal(y.values.view(torch.uint8), q.values.view(torch.uint8)) and torch.equal(y.scales, q.scales)
    stack = x.contiguous().view(5, 1, K)
    assert torch.equal(cl.rms_norm(stack, g).view(5, K), cl.rms_norm(x, g))


@pytest.mark.parametrize("out", [torch.float32, ref.F8])
def test_norm_of_rows_that_are_not_finite(out):
    x = torch.ones((5, 300), device="cuda")
    x[0, 3], x[1, 200], x[2] = float("nan"), float("inf"), 0.0
    x[3] *= 1e-30
    y = cl.rms_norm(x, eps=1e-6, dtype=out)
    v = cl.f8_dequantize(y) if out == ref.F8 else y
    assert v[0].isnan().all() and v[4].sub(1).abs().max() < 2.0 ** -4 and (v[2] == 0).all()
    # an infinite mean: what is finite becomes zero, Inf NaN (in 8 bits its block)
    nan = torch.zeros(300, dtype=torch.bool, device="cuda")
    nan[128:256 if out == ref.F8 else 256] = True
    assert torch.equal(v[1].isnan(), nan if out == ref.F8 else torch.arange(300, device="cuda") == 200)
    assert (v[1][~v[1].isnan()] == 0).all() and torch.allclose(v[3], torch.full((300,), 1e-27, device="cuda"), rtol=0.07)


# --------------------------------------------------------------------------- #
# products
# --------------------------------------------------------------------------- #
# batch, outputs, K
SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 31), (3, 100, 513), (15, 33, 127), (16, 64, 512), (17, 130, 640), (33, 48, 1000), (64, 128, 256), (65, 96, 4100),
          (130, 259, 384), (1, 4096, 1030), (8, 1000, 4096), (300, 257, 2050), (513, 300, 700), (5, 20, 9000)]


def weights(rng, rows, K):
    w = torch.from_numpy((rng.standard_normal((rows, K)) * 2.0 ** rng.integers(-3, 4, (rows, 1)) * 0.02).astype(np.float32)).cuda()
    return cl.f8_quantize(w, 128)


def operands(rng, B, M, K, dtype, act):
    w = cl.f8_gated(weights(rng, M, K), weights(rng, M, K)) if act == "gated" else weights(rng, M, K)
    x = spread(rng, (B, K), dtype)
    return x, w, ref.quantised(x.double().cpu().numpy()), ref.stand_for(w)


@pytest.mark.parametrize("act", ["none", "relu", "gated"])
@pytest.mark.parametrize("B,M,K", SHAPES)
def test_product(B, M, K, act):
    rng = np.random.default_rng(B + M + K)
    for i, dtype in enumerate(ref.DTYPES):
        x, w, xq, wq = operands(rng, B, M, K, dtype, act)
        bias = rng.standard_normal(len(wq)).astype(np.float32) if i != 1 else None
        bd = None if bias is None else torch.from_numpy(bias).cuda()
        y = cl.f8_fc_forward(w, x, bd, act=act)
        assert y.dtype == dtype and y.shape == (B, M)
        whole, most = ref.product(xq, wq, bias, act), ref.product(xq, wq, bias, act, ref.eights(xq, wq))
        ref.assert_within(y, *(whole if dtype == torch.float32 else most), (B, M, K, dtype))
        assert torch.equal(y, cl.f8_fc_forward(w, x, bd, act=act))                        # run to run
        # quantised beforehand, and other output types
        q = cl.f8_quantize(x)
        for out in ref.DTYPES + [ref.F8]:
            z = cl.f8_fc_forward(w, q, bd, act=act, dtype=out)
            if out == ref.F8:
                ref.assert_f8_within(z, *whole, (B, M, K, dtype))
            else:
                assert z.dtype == out
                ref.assert_within(z, *(whole if out == torch.float32 else most), (B, M, K, dtype, out))
        z = cl.f8_fc_forward(w, x, bd, act=act, dtype=ref.F8)
        ref.assert_f8_within(z, *whole, (B, M, K, dtype))
