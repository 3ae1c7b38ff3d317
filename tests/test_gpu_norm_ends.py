"""Where rows of a norm end: inside 16 bytes of numbers, at any distance from each other among numbers that are none, in place, over several wavefronts, longer than what stays in
registers."""
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


def strided(rows, K, dtype, seed, gap):
    """Rows of K numbers, gap NaN behind each and in front of the first."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    room = torch.full((rows * (K + gap) + gap,), float("nan"), dtype=dtype, device="cuda")
    view = room[gap:].view(rows, K + gap)[:, :K]
    view.copy_(torch.randn((rows, K), generator=g, device="cuda"))
    return room, view


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("rows,K", [(9, 1), (3, 2), (40, 3), (17, 4), (33, 5), (19, 7), (19, 8), (70, 9), (200000, 11), (21, 15), (5, 69), (300, 129), (2, 1023), (900, 1025), (7, 8197), (3, 20003), (2, 70001)])
def test_the_ends_of_rows(rows, K, dtype):
    room, x = strided(rows, K, dtype, K, 3)
    _, r = strided(rows, K, dtype, K + 1, 5)
    before = room.clone()
    gain = torch.randn(K, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    y, total = cl.rms_norm(x, gain, 1e-5, residual=r, dtype=torch.float32)
    assert torch.equal(total, (x.float() + r.float()).to(dtype)) and torch.equal(room.view(torch.uint8), before.view(torch.uint8))
    h = total.double()
    want = h / (h.square().mean(1, keepdim=True) + 1e-5).sqrt() * gain.double()
    # (a sum of K squares in 32 bits, any order: within K steps of half a last place, halved by the root; root, quotient, two products and their stored values: six more)
    assert bool(((y.double() - want).abs() <= want.abs() * (0.5 * min(K, 64 + 8 + K / 1024 + 24) + 6) * 2.0 ** -24).all())
    same = cl.rms_norm(x.contiguous(), gain, 1e-5, residual=r.contiguous(), dtype=torch.float32)
    assert torch.equal(same[0], y) and torch.equal(same[1], total)
    q, _ = cl.rms_norm(x, gain, 1e-5, residual=r, dtype=ref.F8)
    z = cl.f8_quantize(y)
    assert torch.equal(q.values.view(torch.uint8), z.values.view(torch.uint8)) and torch.equal(q.scales, z.scales)
    # the sum where X was, the output where X was; what is beside the rows stays
    out, again = cl.rms_norm(x, gain, 1e-5, residual=r, sum_out=x)
    assert again.data_ptr() == x.data_ptr() and torch.equal(x, total) and torch.equal(out, y.to(dtype))
    want = cl.rms_norm(x, gain, 1e-5)
    cl.rms_norm(x, gain, 1e-5, out=x)
    assert torch.equal(x, want)
    beside = torch.ones_like(room, dtype=torch.bool)
    beside[3:].view(rows, K + 3)[:, :K] = False
    assert bool(room[beside].isnan().all())
