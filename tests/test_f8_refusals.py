"""The entry points of the 8-bit operators refuse what they cannot serve, before anything is launched: none of this needs a GPU.  And the plain forms that the GPU
tests compare with (f8_ref) against what the format's definition says."""
import ctypes as C

import numpy as np
import pytest
import torch

import f8_ref as ref
from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EINVAL, CL_EUNSUPPORTED, CL_OK, F8Input, F8Matrix, NormCall

P = C.c_void_p(4096)              # an aligned address that no refused call touches
ODD = C.c_void_p(4097)
Y = C.c_void_p(1 << 20)             # another
NAN, INF = float("nan"), float("inf")


def test_quantise():
    f, back = binding.lib().cl_eight_quantize, binding.lib().cl_eight_dequantize
    for args in [(None, 0, 64, 1, 64, 1, P, P, None), (P, 0, 64, 1, 64, 1, None, P, None), (P, 0, 64, 1, 64, 1, P, None, None), (P, 3, 64, 1, 64, 1, P, P, None),
                 (P, 4, 64, 1, 64, 1, P, P, None), (P, 0, 64, -1, 64, 1, P, P, None), (P, 0, 64, 1, 0, 1, P, P, None), (P, 0, 63, 2, 64, 1, P, P, None),
                 (P, 0, 64, 1, 64, 1, ODD, P, None), (P, 0, 64, 1, 64, 1, P, C.c_void_p(4096 + 8), None), (ODD, 1, 64, 1, 64, 1, P, P, None),
                 (P, 0, 64, 1, 64, 0, P, P, None), (P, 0, 64, 1, 64, 64, P, P, None)]:
        assert f(*args) == CL_EINVAL, args
        assert back(args[6], args[7], args[3], args[4], args[5], args[0], args[1], args[2], None) == CL_EINVAL, args
    assert f(P, 0, 1 << 25, 1, 1 << 25, 1, P, P, None) == CL_EUNSUPPORTED
    assert f(None, 0, 64, 0, 64, 1, None, None, None) == CL_OK and f(None, 0, 64, 0, 64, 128, None, None, None) == CL_OK            # no rows


def test_norm():
    L = binding.lib()

    def call(**kw):
        base = dict(d_X=4096, d_residual=None, d_gain=None, d_sum=None, d_Y=4096, d_y_scales=None, x_stride=64, residual_stride=64, sum_stride=64, y_stride=64, rows=2,
                    K=64, type=1, gain_type=0, y_type=1, eps=1e-6)
        return L.cl_rms_norm(NormCall(**{**base, **kw}), None)

    for kw in (dict(d_X=None), dict(d_Y=None), dict(type=3), dict(type=4), dict(y_type=3), dict(y_type=5), dict(rows=-1), dict(K=0), dict(x_stride=63), dict(y_stride=63),
               dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(d_X=4097), dict(d_Y=4097), dict(d_residual=4096), dict(d_residual=4096, d_sum=8192, residual_stride=63),
               dict(d_residual=4096, d_sum=8192, sum_stride=63), dict(d_residual=4097, d_sum=8192), dict(d_residual=8192, d_sum=4096), dict(d_gain=4096, gain_type=2),
               dict(d_gain=4098, gain_type=0), dict(d_gain=4097, gain_type=1), dict(y_type=4), dict(y_type=4, d_y_scales=4104), dict(y_type=4, d_Y=4104, d_y_scales=4096)):
        assert call(**kw) == CL_EINVAL, kw
    # in place, with elements elsewhere
    for kw in (dict(y_type=0), dict(y_type=2), dict(y_stride=65), dict(y_type=4, d_y_scales=8192), dict(d_Y=12288, d_residual=8192, d_sum=4096, sum_stride=65),
               dict(d_Y=12288, d_residual=8192, d_sum=8192, residual_stride=70), dict(d_X=12288, d_residual=4096, d_sum=8192, y_type=0)):
        assert call(**kw) == CL_EINVAL, kw
    assert call(K=(1 << 24) + 1, x_stride=1 << 25, y_stride=1 << 25) == CL_EUNSUPPORTED
    assert L.cl_rms_norm(None, None) == CL_EINVAL
    assert call(rows=0, d_X=None, d_Y=None) == CL_OK


def test_product():
    L = binding.lib()
    n = C.c_size_t(0)
    W, X = F8Matrix(4096, 4096, 64, 200), F8Input(4096, None, 0, 200)
    assert L.cl_eight_fc_workspace_bytes(W, 30000, 0, 0, 0, n) == CL_OK and n.value >= 30000 * (256 + 16)
    assert L.cl_eight_fc_workspace_bytes(W, 30000, 4, 0, 0, n) == CL_OK and n.value == 0
    for bad in (F8Matrix(4096, 4096, 0, 200), F8Matrix(4096, 4096, 64, 0)):
        assert L.cl_eight_fc_workspace_bytes(bad, 3, 0, 0, 0, n) == CL_EINVAL
    for args in ((-1, 0, 0, 0), (1, 3, 0, 0), (1, 0, 3, 0), (1, 0, 0, 3)):
        assert L.cl_eight_fc_workspace_bytes(W, *args, n) == CL_EINVAL, args
    assert L.cl_eight_fc_workspace_bytes(W, 1, 0, 0, 0, None) == CL_EINVAL and L.cl_eight_fc_workspace_bytes(None, 1, 0, 0, 0, n) == CL_EINVAL
    assert L.cl_eight_fc_workspace_bytes(F8Matrix(4096, 4096, 2**31 - 1, 200), 1, 0, 0, 0, n) == CL_EUNSUPPORTED
    big = 1 << 24

    def call(W=W, X=X, y=Y, ys=P, y_type=0, batch=30000, act=0, ws=P, ws_bytes=big):
        return L.cl_eight_fc_forward(W, X, None, y, ys, y_type, batch, act, ws, ws_bytes, None)

    assert call(W=None) == CL_EINVAL and call(X=None) == CL_EINVAL and call(y=None) == CL_EINVAL
    assert call(y_type=3) == CL_EINVAL and call(act=5) == CL_EINVAL and call(batch=-1) == CL_EINVAL and call(y=ODD) == CL_EINVAL
    assert call(y_type=4, ys=None) == CL_EINVAL and call(y_type=4, y=C.c_void_p(4104)) == CL_EINVAL and call(y_type=4, ys=C.c_void_p(4104)) == CL_EINVAL
    assert call(W=F8Matrix(4096, 4096, 63, 200), act=2) == CL_EINVAL
    assert call(W=F8Matrix(4104, 4096, 64, 200)) == CL_EINVAL and call(W=F8Matrix(4096, 4104, 64, 200)) == CL_EINVAL
    assert call(W=F8Matrix(None, 4096, 64, 200)) == CL_EINVAL and call(W=F8Matrix(4096, None, 64, 200)) == CL_EINVAL
    assert call(W=F8Matrix(4096, 4096, 64, (1 << 24) + 1)) == CL_EUNSUPPORTED
    assert call(X=F8Input(4096, None, 0, 199)) == CL_EINVAL and call(X=F8Input(4096, None, 4, 0)) == CL_EINVAL and call(X=F8Input(4098, None, 0, 200)) == CL_EINVAL
    assert call(X=F8Input(4104, 4096, 4, 0)) == CL_EINVAL and call(X=F8Input(4096, 4104, 4, 0)) == CL_EINVAL
    assert call(ws=None) == CL_EINVAL and call(ws_bytes=16) == CL_EINVAL and call(ws=C.c_void_p(4096 + 16)) == CL_EINVAL
    assert call(y=P) == CL_EINVAL and "one" in L.cl_last_error().decode()             # the input's own place
    assert call(batch=0, y=None, ws=None, ws_bytes=0) == CL_OK


def test_the_plain_quantiser():
    rng = np.random.default_rng(0)
    # against torch's own conversion, and that no 8-bit value is nearer
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 8, 4000), [448, 463.9, 0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17, 19]]).clip(-463.9, 463.9)
    assert np.array_equal(ref.e4m3(x.astype(np.float32)), torch.from_numpy(x.astype(np.float32)).to(ref.F8).double().numpy())
    every = torch.arange(256, dtype=torch.uint8).view(ref.F8).double().numpy()
    every = every[~np.isnan(every)]
    assert np.array_equal(np.abs(ref.e4m3(x) - x), np.abs(x[:, None] - every).min(axis=1))
    x = (rng.standard_normal((300, 200)) * 2.0 ** rng.integers(-20, 20, (300, 200))).astype(np.float32)
    for block_rows in (1, 128):
        codes, scales = ref.quantise(x, block_rows)
        assert codes.shape == (300, 256) and scales.shape == (-(-300 // block_rows), 2) and (codes[:, 200:] == 0).all()
        assert np.abs(codes).max() == 448 and (np.abs(ref.values(codes, scales, 200, block_rows) - x) <= np.abs(x) * 2.0 ** -4 * 1.001 + np.repeat(np.repeat(scales, block_rows, 0)[:300], 128, 1)[:, :200] * 2.0 ** -9.99).all()
    x[3, 5] = np.nan
    assert np.isnan(ref.quantise(x)[1][3, 0]) and (ref.quantise(x)[0][3, :128] == 0).all() and np.isnan(ref.quantise(x, 128)[1][0, 0])


@pytest.mark.parametrize("act", ["none", "relu", "gated"])
def test_the_bounds_of_a_product(act):
    rng = np.random.default_rng(1)
    x, w = ref.quantised(rng.standard_normal((20, 300))), ref.quantised(rng.standard_normal((30, 300)))
    want, err = ref.product(x, w, None, act)
    acc, cut = np.zeros((20, 30), np.float32), np.zeros((20, 30))
    for k in range(0, 300, 8):
        terms = x[:, None, k:k + 8] * w[None, :, k:k + 8]
        for j in range(terms.shape[2]):
            acc += terms[:, :, j].astype(np.float32)
        unit = 2.0 ** (np.floor(np.log2(np.abs(terms).max(2, keepdims=True) + 1e-300)) - 13)
        cut += (np.trunc(terms / unit) * unit).sum(2)

    def after(v):
        if act == "gated":
            return v[:, :15] / (1 + np.exp(-v[:, :15])) * v[:, 15:]
        return np.maximum(v, 0) if act == "relu" else v

    assert (np.abs(after(acc.astype(np.float64)) - want) <= err).all()
    most, loose = ref.product(x, w, None, act, ref.eights(x, w))
    assert np.array_equal(most, want) and (np.abs(after(cut) - want) <= loose).all()
    if act == "none":
        wrong = acc + (x[:, :1] * w[:, 0]).astype(np.float32)          # a term too many is seen
        assert (np.abs(wrong - want) > err).mean() > 0.8 and (np.abs(wrong - want) > loose).mean() > 0.5
