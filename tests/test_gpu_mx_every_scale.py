"""What codes and scales stand for, all of them: sixteen codes under each of the 256 scale bytes, in every type; and products that one such block makes."""
import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


def every():
    """256 rows of a block of all codes, twice, under the row's own scale byte: values fp64."""
    codes = np.zeros((256, 64), np.uint8)
    codes[:, :16] = np.tile(np.arange(0, 16, 2) | np.arange(1, 16, 2) << 4, 2)
    scales = np.zeros((256, 4), np.uint8)
    scales[:, 0] = np.arange(256)
    return cl.MxTensor(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 32), ref.values(codes, scales, 32)


@pytest.mark.parametrize("dtype", ref.DTYPES)
def test_back(dtype):
    q, want = every()
    y = cl.mx_dequantize(q, dtype).cpu()
    want = torch.from_numpy(want).to(torch.float32).to(dtype)            # (at most two bits: fp32 rounds none of them, but to infinity)
    assert torch.equal(y.isnan(), want.isnan()) and y[255].isnan().all() and not y[:255].isnan().any()
    assert torch.equal(y[:255], want[:255])
    assert torch.equal(torch.signbit(y[:255]), torch.signbit(want[:255]))


@pytest.mark.parametrize("other", [7, 60, 127, 190, 250])
def test_products(other):
    q, values = every()
    x, xv = every()
    x.scales[:, 0], xv = other, np.tile(values[other], (256, 1))
    want = xv[:20] @ values.T
    y = cl.mx_fc_forward(q, cl.MxTensor(x.codes[:20], x.scales[:20], 32)).double().cpu().numpy()
    # sums of 32 products; where fp32 holds every product and the sum as ordinary numbers they are exact
    least, most = 0.5 * 2.0 ** (np.arange(255) - 127.0), 6 * 2.0 ** (np.arange(255) - 127.0)
    unit = 2.0 ** (other - 127)
    ok = np.append((least * 0.5 * unit >= 2.0 ** -126) & (most * 6 * unit * 32 < 2.0 ** 128), False)
    assert ok.sum() > 100
    assert np.array_equal(y[:, ok], want[:, ok])
    assert np.isnan(y[:, 255]).all()
