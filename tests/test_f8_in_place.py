"""Conversions to 8 bits and back do not work in place - an element and what it becomes are not in one spot -, and say so before anything is launched: no GPU needed."""
import ctypes as C

import pytest

from paper_1711_00244_amd import binding
from paper_1711_00244_amd.binding import CL_EINVAL

P, Q, R = C.c_void_p(4096), C.c_void_p(8192), C.c_void_p(12288)      # aligned addresses that no refused call touches


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("type_", [0, 1, 2])
def test_one_buffer_for_two(type_, block_rows):
    L = binding.lib()
    for x, values, scales in ((P, P, Q), (P, Q, P), (P, Q, Q), (R, R, R)):
        assert L.cl_eight_quantize(x, type_, 200, 3, 200, block_rows, values, scales, None) == CL_EINVAL and "one" in L.cl_last_error().decode()
        assert L.cl_eight_dequantize(values, scales, 3, 200, block_rows, x, type_, 200, None) == CL_EINVAL and "one" in L.cl_last_error().decode()

