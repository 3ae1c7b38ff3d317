"""8-bit operators side by side: 8-bit outputs beside the quantised fp32 ones, calls from two threads on streams of their own, graphs that share a workspace."""
import threading

import pytest
import torch

import f8_ref as ref
import paper_1711_00244_amd as cl
from paper_1711_00244_amd import feed_forward

pytestmark = pytest.mark.gpu
F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, ref.F8


def draw(B, M, K, gated, seed, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    parts = [cl.f8_quantize(torch.randn((M, K), generator=g, device="cuda") * K ** -0.5, block_rows=128) for _ in range(1 + gated)]
    return cl.f8_gated(*parts) if gated else parts[0], torch.randn((B, K), generator=g, device="cuda").to(dtype)


def same(a, b):
    if isinstance(a, cl.F8Tensor):
        return torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)
    return torch.equal(a, b)


# (shapes whose calls take one form, split alike, for both types: the sums come in one order)
@pytest.mark.parametrize("B,M,K,act", [(5, 333, 1700, "gated"), (9, 500, 2000, "none"), (335, 19, 49, "gated"), (8118, 220, 34, "none"), (100, 1555, 10491, "gated"), (4300, 2200, 260, "gated"),
                                       (5000, 2500, 130, "relu"), (7000, 900, 700, "gated")])
def test_8_bit_outputs_are_the_fp32_ones_quantised(B, M, K, act):
    W, X = draw(B, M, K, act == "gated", M)
    q = cl.f8_quantize(X)
    assert cl.f8_fc_resolved_form(W, B, F8, act, F8) == cl.f8_fc_resolved_form(W, B, F8, act, F32)
    assert same(cl.f8_fc_forward(W, q, act=act, dtype=F8), cl.f8_quantize(cl.f8_fc_forward(W, q, act=act, dtype=F32)))


def test_two_threads_on_streams_of_their_own():
    layers = [feed_forward.synthetic(512, 700, seed=1), feed_forward.synthetic(900, 1300, seed=2)]
    inputs = [[torch.randn((n, layer.width), device="cuda").to(BF16) for n in (1, 40, 700)] for layer in layers]
    want = [[layer.forward(x, x) for x in xs] for layer, xs in zip(layers, inputs)]
    torch.cuda.synchronize()
    wrong, errors = [], []

    def work(n):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for turn in range(20):
                    for i, x in enumerate(inputs[n]):
                        y = layers[n].forward(x, x)
                        if not all(torch.equal(a, b) for a, b in zip(y, want[n][i])):
                            wrong.append((n, turn, i))
        except Exception as e:                                                           # noqa: BLE001 (told below, in the test's own thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and not wrong, (errors, wrong[:5])


def test_two_graphs_with_one_workspace():
    W, X = draw(300, 400, 9000, False, 3, BF16)
    V, Z = draw(200, 300, 6000, True, 4, F16)
    need = max(cl.f8_fc_workspace_bytes(W, 300, BF16), cl.f8_fc_workspace_bytes(V, 200, F16, "gated"))
    assert need
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    calls = [lambda: cl.f8_fc_forward(W, X, workspace=room), lambda: cl.f8_fc_forward(V, Z, act="gated", workspace=room)]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        want = [f().clone() for f in calls]
        stream.synchronize()
        graphs, out = [], []
        for f in calls:
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=stream):
                out.append(f())
        for turn in range(6):
            room.fill_(255)
            for n in (turn % 2, 1 - turn % 2):
                graphs[n].replay()
            assert torch.equal(calls[turn % 2](), want[turn % 2])                       # (the program's own work between)
            stream.synchronize()
            for n in range(2):
                assert torch.equal(out[n], want[n])
                out[n].zero_()
