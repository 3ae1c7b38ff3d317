"""Calls with the workspace of a larger batch: a product that would split its sums, and has no room for the parts, runs without."""
import pytest
import torch

import mx_ref as ref
import paper_1711_00244_amd as cl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,largest,batches", [(4096, 9216, 256, (1, 32, 64, 128, 192, 255, 256)), (962, 7400, 700, (33, 100, 265, 500)), (2048, 5000, 300, (60, 128, 250, 256))])
def test_the_workspace_of_the_largest_batch_serves_all(M, K, largest, batches):
    g = torch.Generator(device="cuda").manual_seed(M)
    W = cl.mx_quantize(torch.randn((M, K), generator=g, device="cuda") * 0.05)
    wq = cl.mx_dequantize(W).double()
    need = cl.mx_fc_workspace_bytes(W, largest, torch.float32)
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    assert need > 0
    short = 0
    for batch in batches:
        X = torch.randn((batch, K), generator=g, device="cuda")
        short += cl.mx_fc_workspace_bytes(W, batch, torch.float32) > need
        y = cl.mx_fc_forward(W, X, workspace=room[:need])
        xq = cl.mx_dequantize(cl.mx_quantize(X)).double()
        want, size = xq @ wq.T, xq.abs() @ wq.abs().T
        # mx_ref's bound of an fp32 sum of K terms in any order
        err = (K + 4) * 2.0 ** -23 * size
        bound = err + ref.HALF_ULP[torch.float32] * (want.abs() + err)
        assert bool(((y.double() - want).abs() <= bound).all()), batch
        assert torch.equal(y, cl.mx_fc_forward(W, X, workspace=room[:need])) and bool((room[need:] == 255).all())
        # rows that are there in 4 bits need no workspace at all
        z = cl.mx_fc_forward(W, cl.mx_quantize(X), dtype=torch.float32, workspace=room[:0])
        assert bool(((z.double() - want).abs() <= bound).all()), batch
    assert short > 0                                         # (what this is about is among them)
    codes = 17 * cl.mx_row_blocks(K) * largest
    with pytest.raises(cl.CLError):
        cl.mx_fc_forward(W, torch.zeros((largest, K), device="cuda"), workspace=room[:codes // 512 * 256])
