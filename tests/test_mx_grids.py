"""Products whose launch would have 2^32 threads or more along an axis are refused as what they are, before anything is launched - the quantisation of X
and the lists of the experts among it -, and already where the workspace is sized.  None of this needs a GPU."""
import ctypes as C

import pytest

from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EUNSUPPORTED, CL_OK, MxExpertsCall, MxInput, MxMatrix

P = C.c_void_p(4096)              # an aligned address that no refused call touches
ALL = (1 << 48)


@pytest.mark.parametrize("M,K,batch", [(1, 1, 1 << 30), (64, 8, (1 << 30) + 5), (128, 64, (1 << 31) - 1), ((1 << 31) - 1, 8, 1), (1 << 30, 64, 40), ((1 << 31) - 16, 200, 1 << 20)])
def test_product(M, K, batch):
    L, n = binding.lib(), C.c_size_t(0)
    W = MxMatrix(4096, 4096, M, K)
    for x_type in (0, 3):
        assert L.cl_mx_fc_workspace_bytes(W, batch, x_type, n) == CL_EUNSUPPORTED
        assert L.cl_mx_fc_forward(W, MxInput(4096, 4096, x_type, K), None, P, 0, batch, 0, P, ALL, None) == CL_EUNSUPPORTED


@pytest.mark.parametrize("M,K,tokens,k,experts", [(64, 8, 1 << 30, 1, 2), (1 << 20, 8, 1 << 25, 2, 2), ((1 << 31) - 1, 8, 1, 8, 64)])
@pytest.mark.parametrize("x_per_pair", [0, 1])
def test_experts(M, K, tokens, k, experts, x_per_pair):
    L, n = binding.lib(), C.c_size_t(0)
    W = MxMatrix(4096, 4096, M, K)
    for weights in (None, 4096):
        for lists in (None, 4096):
            call = MxExpertsCall(tokens, k, 4096, weights, None, lists, 0, x_per_pair)
            for x_type in (0, 3):
                assert L.cl_mx_experts_workspace_bytes(W, experts, call, x_type, n) == CL_EUNSUPPORTED
                assert L.cl_mx_experts_forward(W, experts, MxInput(4096, 4096, x_type, K), call, P, 0, P, ALL, None) == CL_EUNSUPPORTED


def test_what_fits_is_sized():
    L, n = binding.lib(), C.c_size_t(0)
    assert L.cl_mx_fc_workspace_bytes(MxMatrix(4096, 4096, 64, 8), 1 << 29, 0, n) == CL_OK and n.value >= 1 << 35
    assert L.cl_mx_fc_workspace_bytes(MxMatrix(4096, 4096, 1 << 26, 8192), 1, 0, n) == CL_OK
