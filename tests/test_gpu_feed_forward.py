"""A gated feed-forward block in 8 bits (paper_1711_00244_amd.feed_forward): its steps against the plain forms (f8_ref), the whole as one call, recorded call and refused call, and as
the shared expert of a layer of routed experts."""
import json
import subprocess
import sys

import numpy as np
import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl
from paper_1711_00244_amd import experts as ex
from paper_1711_00244_amd import feed_forward as ff

pytestmark = pytest.mark.gpu
F8 = ref.F8


def tokens(T, width, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((T, width), generator=g, device="cuda").to(dtype), torch.randn((T, width), generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("T,width,hidden", [(1, 130, 34), (19, 256, 700), (200, 300, 129), (700, 136, 1000)])
def test_layer_against_its_steps(T, width, hidden, dtype):
    layer = ff.synthetic(width, hidden, seed=T)
    X, residual = tokens(T, width, dtype)
    Y, total = layer.forward(X, residual)
    h = (X.float() + residual.float()).to(dtype)
    assert torch.equal(total, h) and Y.dtype == dtype and Y.shape == (T, width)
    # each step from what the one before it made: the norm, the gated product, the second matrix
    normed = cl.rms_norm(X, layer.gain, layer.eps, residual=residual, dtype=F8)[0]
    ref.assert_f8_within(normed, *ref.norm(h.double().cpu().numpy(), layer.gain.double().cpu().numpy(), layer.eps))
    mid = cl.f8_fc_forward(layer.up, normed, act="gated", dtype=F8)
    x, up = ref.stand_for(normed), ref.stand_for(layer.up)
    ref.assert_f8_within(mid, *ref.product(x, up, None, "gated"))
    x, down = ref.stand_for(mid), ref.stand_for(layer.down)
    ref.assert_within(Y, *ref.product(x, down, None, "none", None if dtype == torch.float32 else ref.eights(x, down)))
    alone = layer.forward(h)
    assert torch.equal(alone, Y)


@pytest.mark.parametrize("T", [1, 90, 1500])
def test_layer_recorded(T):
    layer = ff.synthetic(256, 640, seed=5)
    X, residual = tokens(T, 256, torch.bfloat16)
    layer.forward(X, residual)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, total = layer.forward(X, residual)
    for seed in (2, 3, 4):
        a, b = tokens(T, 256, torch.bfloat16, seed)
        X.copy_(a)
        residual.copy_(b)
        graph.replay()
        got = Y.clone(), total.clone()
        torch.cuda.synchronize()
        again = layer.forward(X, residual)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_no_tokens_and_refusals():
    layer = ff.synthetic(256, 128)
    X = torch.empty((0, 256), device="cuda")
    assert layer.forward(X).shape == (0, 256) and layer.forward(X, X)[1].shape == (0, 256)
    other = ff.synthetic(256, 384)
    for bad in (lambda: ff.GatedLayer(layer.up, other.down), lambda: ff.GatedLayer(layer.down, layer.up), lambda: ff.GatedLayer(layer.up, layer.down, torch.ones(255, device="cuda")),
                lambda: layer.forward(torch.zeros((3, 255), device="cuda")), lambda: layer.forward(torch.zeros((3, 256), device="cuda"), torch.zeros((2, 256), device="cuda"))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("T", [1, 90])
def test_shared_expert_in_8_bits(T):
    layer = ex.synthetic(16, 256, 64, 2, shared=False, seed=5)
    block = ff.synthetic(256, 384, seed=6)
    both = ex.ExpertLayer(layer.router, layer.up, layer.down, 2, (block.up, block.down))
    X = tokens(T, 256, torch.float32)[0]
    want = layer.forward(X) + cl.f8_fc_forward(block.down, cl.f8_fc_forward(block.up, X, act="gated", dtype=F8), dtype=torch.float32)
    assert torch.equal(both.forward(X), want)
    with pytest.raises(ValueError):
        ex.ExpertLayer(layer.router, layer.up, layer.down, 2, (block.down, block.up))
    with pytest.raises(ValueError):
        wrong = ff.synthetic(160, 384)
        ex.ExpertLayer(layer.router, layer.up, layer.down, 2, (wrong.up, wrong.down))


def test_command():
    out = subprocess.run([sys.executable, "-m", "paper_1711_00244_amd.feed_forward", "--width", "256", "--hidden", "512", "--tokens", "3", "70", "--steps", "2"], capture_output=True, text=True,
                         check=True, timeout=100).stdout
    rows = [json.loads(line) for line in out.splitlines() if line.startswith("{")]
    assert [r["tokens"] for r in rows] == [3, 70] and all(np.isfinite(r["ms"]) and r["ms"] > 0 for r in rows)
