"""The scratch that is asked for a batch is enough for smaller ones, 8-bit products that do not fit a grid are refused as what they are, and sizes beyond 32 bits are.
Sizes and refusals only: none of this needs a GPU, and where there is one the calls that would be launched are left out."""
import ctypes as C
import random
from types import SimpleNamespace

import pytest
import torch

import paper_1711_00244_amd as cl
from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EHIP, CL_EINVAL, CL_EUNSUPPORTED, CL_OK, F8Input, F8Matrix

P = C.c_void_p(4096)              # an aligned address that no refused call touches
Y = C.c_void_p(1 << 20)
BIG = 1 << 32


def need(M, K, batch, x_type, y_type, act):
    n = C.c_size_t(0)
    assert binding.lib().cl_eight_fc_workspace_bytes(F8Matrix(None, None, M, K), batch, x_type, y_type, act, n) == CL_OK
    return n.value


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would be launched, with addresses that are none")
def test_enough_for_smaller_batches():
    """Without a GPU a call that passes all checks fails at its first launch; one whose workspace is too small before."""
    L, rng = binding.lib(), random.Random(4)
    W = lambda M, K: F8Matrix(4096, 4096, M, K)  # noqa: E731
    refused = 0
    for _ in range(60):
        M, K, batch = 2 * int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 14.6)), int(2 ** rng.uniform(0, 13))
        for act in (0, 2):
            for x_type, y_type in ((0, 0), (1, 1), (0, 4), (1, 4), (4, 4), (4, 2)):
                n = need(M, K, batch, x_type, y_type, act)
                smaller = sorted({max(1, batch - d) for d in (0, 1, 15, 16, 17)} | {rng.randint(1, batch) for _ in range(6)} | {1, batch // 2 + 1, batch // 8 + 1})
                for b in smaller:
                    rc = L.cl_eight_fc_forward(W(M, K), F8Input(4096, 4096, x_type, K), None, Y, P, y_type, b, act, P if n else None, n, None)
                    assert rc == CL_EHIP, (M, K, batch, b, act, x_type, y_type, n, rc, binding.lib().cl_last_error())
                if batch > 256 and x_type != 4:
                    # room for half of X's values only
                    rc = L.cl_eight_fc_forward(W(M, K), F8Input(4096, 4096, x_type, K), None, Y, P, y_type, batch, act, P, batch * K // 2 // 256 * 256, None)
                    assert rc == CL_EINVAL
                    refused += 1
    assert refused > 100


@pytest.mark.parametrize("M,K,batch", [(1 << 30, 64, 40000), ((1 << 31) - 1024, 200, 1 << 20)])
def test_products_that_do_not_fit_a_grid(M, K, batch):
    L, n = binding.lib(), C.c_size_t(0)
    for x_type in (0, 4):
        assert L.cl_eight_fc_workspace_bytes(F8Matrix(4096, 4096, M, K), batch, x_type, 0, 0, n) == CL_EUNSUPPORTED
        assert L.cl_eight_fc_forward(F8Matrix(4096, 4096, M, K), F8Input(4096, 4096, x_type, K), None, Y, P, 0, batch, 0, P, 1 << 60, None) == CL_EUNSUPPORTED


def test_no_rows():
    for x_type in (0, 1, 2, 4):
        for y_type in (0, 1, 2, 4):
            for act in (0, 1, 2):
                assert need(256, 256, 0, x_type, y_type, act) == 0 and need(4096, 20000, 0, x_type, y_type, act) == 0


def test_sizes_beyond_32_bits():
    W = SimpleNamespace(shape=(64, 200), K=200)
    for ask in (lambda: cl.f8_fc_workspace_bytes(W, BIG + 3), lambda: cl.f8_fc_resolved_form(W, BIG + 3), lambda: cl.f8_fc_resolved_form(SimpleNamespace(shape=(BIG + 64, 200), K=200), 3)):
        with pytest.raises(ValueError):
            ask()
    assert cl.f8_fc_workspace_bytes(W, 30000) > 0 and cl.f8_fc_resolved_form(W, 3) == ("few numbers", 1)
