"""Which form a product with 4-bit matrices takes can be asked without a GPU: the forms that the tests on one name are these."""
import ctypes as C

import pytest

from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EINVAL, CL_EUNSUPPORTED, CL_OK, MX_FORMS, MxExpertsCall, MxMatrix


def fc_form(M, K, batch, x_type=0):
    form, splits = C.c_int32(-1), C.c_int32(-1)
    assert binding.lib().cl_mx_fc_resolved_form(MxMatrix(None, None, M, K), batch, x_type, form, splits) == CL_OK
    return MX_FORMS[form.value], splits.value


def experts_form(M, K, experts, tokens, k, x_type=0, weighted=True, lists=False, x_per_pair=0):
    form = C.c_int32(-1)
    call = MxExpertsCall(tokens, k, None, 256 if weighted else None, None, 256 if lists else None, 0, x_per_pair)
    assert binding.lib().cl_mx_experts_resolved_form(MxMatrix(None, None, M, K), experts, call, x_type, form) == CL_OK
    return MX_FORMS[form.value]


def test_products():
    assert fc_form(4096, 9216, 1) == ("few", 1) and fc_form(4096, 9216, 1, 3) == ("rows", 1)        # (rows in 4 bits need no quantisation)
    assert fc_form(4096, 9216, 256)[0] == "tile 64" and fc_form(4096, 25088, 4096) == ("tile 256", 1)
    assert {fc_form(M, K, b)[1] for M, K, b in ((265, 7400, 265), (962, 7400, 265), (438, 6681, 257), (400, 8200, 250))} <= {1, 2, 4, 8}


def test_experts():
    assert experts_form(1024, 4096, 64, 1, 8) == "few" and experts_form(2048, 4096, 64, 8192, 4) == "tile 256"
    assert experts_form(1024, 4096, 64, 1, 8, x_type=3) != "few"


def test_refusals():
    L, n, form = binding.lib(), C.c_int32(0), C.c_int32(0)
    W = MxMatrix(None, None, 64, 200)
    assert L.cl_mx_fc_resolved_form(W, 1, 0, None, n) == CL_EINVAL and L.cl_mx_fc_resolved_form(W, 1, 0, form, None) == CL_EINVAL
    assert L.cl_mx_fc_resolved_form(None, 1, 0, form, n) == CL_EINVAL and L.cl_mx_fc_resolved_form(W, -1, 0, form, n) == CL_EINVAL
    assert L.cl_mx_fc_resolved_form(W, 1, 9, form, n) == CL_EINVAL and L.cl_mx_fc_resolved_form(MxMatrix(None, None, 1, 1), 1 << 30, 0, form, n) == CL_EUNSUPPORTED
    call = MxExpertsCall(4, 2, None, None, None, None, 0, 0)
    assert L.cl_mx_experts_resolved_form(W, 8, None, 0, form) == CL_EINVAL and L.cl_mx_experts_resolved_form(W, 8, call, 0, None) == CL_EINVAL
    assert L.cl_mx_experts_resolved_form(W, 0, call, 0, form) == CL_EINVAL and L.cl_mx_experts_resolved_form(W, 1025, call, 0, form) == CL_EUNSUPPORTED


@pytest.mark.parametrize("batch", [0, 1, 17, 300, 5000])
def test_forms_are_named(batch):
    for M, K in ((1, 1), (64, 200), (4096, 25088)):
        assert fc_form(M, K, batch)[0] in MX_FORMS and experts_form(M, K, 8, batch, 2) in MX_FORMS
