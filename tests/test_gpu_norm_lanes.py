"""The norm's result does not depend on the type that it is stored in: numbers of rows between which the kernel's launch changes, and lengths of rows that are no whole blocks of 128."""
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu
F32, BF16, F16 = ref.DTYPES


@pytest.mark.parametrize("rows,K,dtype", [(40000, 130, BF16), (40000, 130, F16), (8300, 1000, BF16), (2860, 2900, F16), (20000, 130, F32), (62000, 130, BF16), (32000, 130, F32), (70000, 69, BF16)])
def test_every_type_has_the_same_result(rows, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(K)
    x, r = (torch.randn((rows, K), generator=g, device="cuda").to(dtype) for _ in range(2))
    gain = 1 + 0.3 * torch.randn(K, generator=g, device="cuda")
    for residual in (None, r):
        run = lambda out: cl.rms_norm(x, gain, 1e-5, residual=residual, dtype=out) if residual is None else cl.rms_norm(x, gain, 1e-5, residual=residual, dtype=out)[0]  # noqa: E731
        y = run(F32)
        for out in (BF16, F16):
            assert torch.equal(run(out), y.to(out))
        q, want = run(ref.F8), cl.f8_quantize(y)
        assert torch.equal(q.scales, want.scales) and torch.equal(q.values.view(torch.uint8), want.values.view(torch.uint8))
