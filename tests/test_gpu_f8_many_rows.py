"""More rows than one launch of the 8-bit conversions and of the norm has threads for: the rows on both sides of where a piece ends against calls of those alone."""
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, ref.F8


def same(q, rows, want):
    return torch.equal(q.values[rows].view(torch.uint8), want.values.view(torch.uint8)) and torch.equal(q.scales[rows], want.scales)


def test_conversions():
    # (2^30 units of 16 bytes of numbers, sixteen to a block)
    piece = 1 << 26
    x = torch.randn((piece + 5000, 3), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=BF16)
    q = cl.f8_quantize(x)
    y = cl.f8_dequantize(q, BF16)
    for rows in (slice(0, 3000), slice(piece - 3000, piece + 3000), slice(len(x) - 3000, len(x))):
        want = cl.f8_quantize(x[rows])
        assert same(q, rows, want) and torch.equal(y[rows], cl.f8_dequantize(want, BF16))


@pytest.mark.parametrize("out", [BF16, F8])
def test_norm(out):
    # (2^32 threads, sixteen to a row)
    piece = (2**32 - 1) // 256 * 16
    rows = piece + 5000 if out == BF16 else (1 << 26) + 5000
    x = torch.randn((rows, 2), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda", dtype=BF16)
    y, total = cl.rms_norm(x, residual=x, dtype=out)
    for part in (slice(0, 3000), slice(min(piece, rows) - 6000, min(piece, rows) + 3000), slice(rows - 3000, rows)):
        want, added = cl.rms_norm(x[part], residual=x[part], dtype=out)
        assert torch.equal(total[part], added) and (torch.equal(y[part], want) if out == BF16 else same(y, part, want))
