"""The entry points of the microscaled 4-bit operators refuse what they cannot serve, before anything is launched: none of this
needs a GPU.  And the plain fp64 forms that the GPU tests compare with (mx_ref) against what the format's definition says."""
import ctypes as C

import numpy as np
import pytest

import mx_ref as ref
from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EINVAL, CL_EUNSUPPORTED, CL_OK, MxExpertsCall, MxInput, MxMatrix, RouteDesc

P = C.c_void_p(4096)              # an aligned address that no refused call touches
ODD = C.c_void_p(4097)


def test_quantise():
    f = binding.lib().cl_mx_quantize
    for args in [(None, 0, 64, 1, 64, P, P, None), (P, 0, 64, 1, 64, None, P, None), (P, 0, 64, 1, 64, P, None, None), (P, 3, 64, 1, 64, P, P, None),
                 (P, 7, 64, 1, 64, P, P, None), (P, 0, 64, -1, 64, P, P, None), (P, 0, 64, 1, 0, P, P, None), (P, 0, 63, 2, 64, P, P, None),
                 (P, 0, 64, 1, 64, ODD, P, None), (P, 0, 64, 1, 64, P, ODD, None), (ODD, 1, 64, 1, 64, P, P, None)]:
        assert f(*args) == CL_EINVAL, args
        assert binding.lib().cl_mx_dequantize(args[5], args[6], args[3], args[4], args[0], args[1], args[2], None) == CL_EINVAL, args
    assert f(P, 0, 1 << 25, 1, 1 << 25, P, P, None) == CL_EUNSUPPORTED
    assert f(None, 0, 64, 0, 64, None, None, None) == CL_OK            # no rows


def test_product():
    L = binding.lib()
    n = C.c_size_t(0)
    W, X = MxMatrix(4096, 4096, 64, 200), MxInput(4096, None, 0, 200)
    assert L.cl_mx_fc_workspace_bytes(W, 30000, 0, n) == CL_OK and n.value >= 30000 * 256 // 32 * 17
    assert L.cl_mx_fc_workspace_bytes(W, 30000, 3, n) == CL_OK and n.value == 0
    assert L.cl_mx_fc_workspace_bytes(W, 3, 0, n) == CL_OK and n.value == 0            # quantised where it is multiplied
    for bad in (MxMatrix(4096, 4096, 0, 200), MxMatrix(4096, 4096, 64, 0)):
        assert L.cl_mx_fc_workspace_bytes(bad, 3, 0, n) == CL_EINVAL
    assert L.cl_mx_fc_workspace_bytes(W, -1, 0, n) == CL_EINVAL and L.cl_mx_fc_workspace_bytes(W, 1, 9, n) == CL_EINVAL
    assert L.cl_mx_fc_workspace_bytes(W, 1, 0, None) == CL_EINVAL and L.cl_mx_fc_workspace_bytes(None, 1, 0, n) == CL_EINVAL
    big = 1 << 23

    def call(W=W, X=X, y=P, y_type=0, batch=30000, act=0, ws=P, ws_bytes=big):
        return L.cl_mx_fc_forward(W, X, None, y, y_type, batch, act, ws, ws_bytes, None)

    assert call(W=None) == CL_EINVAL and call(X=None) == CL_EINVAL and call(y=None) == CL_EINVAL
    assert call(y_type=3) == CL_EINVAL and call(act=5) == CL_EINVAL and call(batch=-1) == CL_EINVAL
    assert call(W=MxMatrix(4096, 4096, 63, 200), act=2) == CL_EINVAL
    assert call(W=MxMatrix(4100, 4096, 64, 200)) == CL_EINVAL and call(W=MxMatrix(4096, 4097, 64, 200)) == CL_EINVAL
    assert call(W=MxMatrix(None, 4096, 64, 200)) == CL_EINVAL
    assert call(W=MxMatrix(4096, 4096, 64, (1 << 24) + 1)) == CL_EUNSUPPORTED
    assert call(X=MxInput(4096, None, 0, 199)) == CL_EINVAL and call(X=MxInput(4096, None, 3, 0)) == CL_EINVAL and call(X=MxInput(4098, None, 0, 200)) == CL_EINVAL
    assert call(ws=None) == CL_EINVAL and call(ws_bytes=16) == CL_EINVAL and call(ws=C.c_void_p(4096 + 16)) == CL_EINVAL
    assert call(batch=0, y=None, ws=None, ws_bytes=0) == CL_OK


def test_route():
    L = binding.lib()

    def call(x=P, ty=0, stride=64, tokens=4, e=P, w=P, **d):
        return L.cl_route_experts(x, ty, stride, None, tokens, RouteDesc(**{**dict(experts=64, k=4, score=0, groups=1, groups_kept=1, group_score=0, renormalize=1, scale=1.0), **d}), e, w, None)

    for kw in (dict(x=None), dict(e=None), dict(w=None), dict(ty=3), dict(stride=63), dict(tokens=-1), dict(experts=0), dict(k=0), dict(k=65), dict(score=2),
               dict(groups=0), dict(groups=3), dict(groups_kept=0), dict(groups=4, groups_kept=5), dict(group_score=2), dict(groups=8, groups_kept=1, k=9)):
        assert call(**kw) == CL_EINVAL, kw
    for kw in (dict(experts=1025), dict(experts=128, stride=128, groups=128), dict(k=33)):
        assert call(**kw) == CL_EUNSUPPORTED, kw
    assert L.cl_route_experts(P, 0, 64, None, 1, None, P, P, None) == CL_EINVAL
    assert call(tokens=0, x=None, e=None, w=None) == CL_OK


def test_experts():
    L = binding.lib()
    n = C.c_size_t(0)
    W, X = MxMatrix(4096, 4096, 64, 200), MxInput(4096, None, 0, 200)
    base = dict(tokens=5000, k=2, d_experts=4096, d_weights=4096, d_bias=None, d_lists=None, act=0, x_per_pair=0)

    def call(W=W, experts=8, X=X, y=P, y_type=0, ws=P, ws_bytes=1 << 24, **c):
        return L.cl_mx_experts_forward(W, experts, X, MxExpertsCall(**{**base, **c}), y, y_type, ws, ws_bytes, None)

    assert L.cl_mx_experts_workspace_bytes(W, 8, MxExpertsCall(**base), 0, n) == CL_OK and n.value > 5000 * 2 * 64 * 4
    assert L.cl_mx_experts_workspace_bytes(W, 8, None, 0, n) == CL_EINVAL
    assert L.cl_expert_lists_bytes(5, 2, 8, n) == CL_OK and n.value >= 4 * (10 + 10)
    assert L.cl_expert_lists_bytes(5, 0, 8, n) == CL_EINVAL and L.cl_expert_lists_bytes(5, 1, 1025, n) == CL_EUNSUPPORTED
    assert L.cl_expert_lists_bytes(1 << 30, 4, 8, n) == CL_EUNSUPPORTED
    assert L.cl_expert_lists(P, 5, 2, 8, None, 1 << 20, None) == CL_EINVAL and L.cl_expert_lists(P, 5, 2, 8, P, 16, None) == CL_EINVAL
    assert L.cl_expert_lists(P, 5, 2, 8, C.c_void_p(4096 + 16), 1 << 20, None) == CL_EINVAL and L.cl_expert_lists(None, 5, 2, 8, P, 1 << 20, None) == CL_EINVAL
    for kw in (dict(W=None), dict(X=None), dict(y=None), dict(experts=0), dict(tokens=-1), dict(k=0), dict(d_experts=None), dict(act=3), dict(ws=None),
               dict(ws_bytes=64), dict(d_lists=4096 + 8), dict(y_type=3)):
        assert call(**kw) == CL_EINVAL, kw
    assert call(experts=1025) == CL_EUNSUPPORTED and call(tokens=1 << 30, k=4) == CL_EUNSUPPORTED
    assert call(tokens=0) == CL_OK


def test_the_plain_quantiser():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 200)) * 2.0 ** rng.integers(-20, 20, (40, 200))
    codes, scales = ref.quantise(x)
    assert codes.shape == (40, 8 * 16) and scales.shape == (40, 8)
    v = ref.values(codes, scales, 200)
    top = np.abs(np.pad(x, ((0, 0), (0, 56))).reshape(40, 8, 32)).max(axis=2)
    scale = 2.0 ** (scales.astype(np.float64) - 127)
    assert ((top[:, :7] / scale[:, :7] >= 4) & (top[:, :7] / scale[:, :7] < 8)).all() and (scales[:, 7] == 0).all()
    # no value of the block's grid is nearer
    every = np.concatenate([ref.GRID, -ref.GRID])
    at = np.repeat(scale, 32, axis=1)[:, :200]
    nearest = np.abs(x[..., None] - every * at[..., None]).min(axis=-1)
    assert np.array_equal(np.abs(x - v), nearest)
    # ties take the even code
    t = np.zeros((1, 32))
    t[0, :8] = [4, .25, .75, 1.25, 1.75, 2.5, 3.5, 5]
    assert ref.quantised(t)[0, :8].tolist() == [4, 0, 1, 1, 2, 2, 4, 4]
    t[0, 3] = np.nan
    assert ref.quantise(t)[1][0, 0] == 255 and np.isnan(ref.quantised(t)).all()


@pytest.mark.parametrize("act", ["none", "relu", "gated"])
def test_the_bound_of_a_product_covers_fp32(act):
    rng = np.random.default_rng(1)
    x, w = ref.quantised(rng.standard_normal((20, 300))), ref.quantised(rng.standard_normal((30, 300)))
    want, err = ref.product(x, w, None, act)
    acc = np.zeros((20, 30), np.float32)
    for j in range(300):
        acc += (x[:, j:j + 1] * w[:, j]).astype(np.float32)
    got = ref.activate(acc.astype(np.float64), act)
    assert (np.abs(got - want) <= err).all()
    if act == "none":                                        # (where an activation is flat, nothing shows)
        wrong = acc + (x[:, :1] * w[:, 0]).astype(np.float32)          # a term too many is seen
        assert (np.abs(wrong - want) > err).mean() > 0.8
