"""Which pairs of matrices a gated block and a shared expert take: what a product would refuse later is refused when the layer is made.  No GPU needed."""
from types import SimpleNamespace

import pytest
import torch

import paper_1711_00244_amd as cl
from paper_1711_00244_amd import experts, feed_forward


def eight(rows, K, block_rows=128, gated=False):
    """An F8Tensor without its data (which its own constructor wants on a GPU)."""
    q = cl.F8Tensor.__new__(cl.F8Tensor)
    q.values, q.scales = torch.empty((rows, cl.f8_row_blocks(K) * 128), dtype=torch.uint8), None
    q.K, q.block_rows, q.gated = K, block_rows, gated
    return q


def four(*shape):
    q = cl.MxTensor.__new__(cl.MxTensor)
    q.codes, q.scales, q.K = torch.empty(shape[:-1] + (cl.mx_row_blocks(shape[-1]) * 16,), dtype=torch.uint8), None, shape[-1]
    return q


TAKEN = [(eight(1400, 256, gated=True), eight(256, 700)), (eight(512, 256), eight(256, 256)), (eight(512, 256, gated=True), eight(256, 256)), (eight(2, 256, gated=True), eight(256, 1))]
REFUSED = [(eight(1400, 256), eight(256, 700)), (eight(2, 256), eight(256, 1)), (eight(512, 256), four(256, 256)), (four(512, 256), eight(256, 256)),
           (eight(512, 256), eight(256, 256, gated=True)), (eight(512, 256, 1), eight(256, 256)), (eight(512, 256), eight(256, 256, 1)), (eight(512, 256), eight(256, 384))]


@pytest.mark.parametrize("up,down", TAKEN)
def test_taken(up, down):
    feed_forward.GatedLayer(up, down)
    experts.ExpertLayer(SimpleNamespace(M=4, K=256), four(4, 64, 256), four(4, 256, 32), 2, (up, down))


@pytest.mark.parametrize("up,down", REFUSED)
def test_refused(up, down):
    with pytest.raises(ValueError):
        feed_forward.GatedLayer(up, down)
    with pytest.raises(ValueError):
        experts.ExpertLayer(SimpleNamespace(M=4, K=256), four(4, 64, 256), four(4, 256, 32), 2, (up, down))


def test_four_bits():
    experts.ExpertLayer(SimpleNamespace(M=4, K=256), four(4, 64, 256), four(4, 256, 32), 2, (four(512, 256), four(256, 256)))
    with pytest.raises(ValueError):
        feed_forward.GatedLayer(four(512, 256), four(256, 256))
