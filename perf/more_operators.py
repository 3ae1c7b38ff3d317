"""Layers in 8-bit floating point with a scale for each block of 128, as measurable cases: quantising weights (a scale to 128 x 128 values) and
activations (a scale to 128 of a row), the root-mean-square norm that adds the residual and hands its output on in 8 bits, the product of an 8-bit
matrix with activations that are quantised on the way, the gated product of a feed-forward block - both projections, the activation and
their product -, and both matrices of such a block, the first's output handed to the second in 8 bits.

Layer shapes are those of workloads.py (AlexNet and VGG-16 fully connected layers) or generic.  What the seed of prepare() changes is everything:
weights, activations, gains.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "f8": 1}
BLOCK = 128                      # elements of a row under one scale
LARGEST = 448.0                  # of the 8-bit format: sign, 4 bits of exponent, 3 of fraction
LEAST = 2.0 ** -126              # of scales
EPS = 1e-6
MOST_FLOPS = 2.0 * 4096 * 4096 * 25088
MOST_VALUES = 4096 * 25088
MOST_NORM = 16384 * 4096


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def _quantise(name, rows, K, dtype, block_rows):
    return dict(name=name, kind="quantise", rows=rows, K=K, dtype=dtype, block_rows=block_rows)


def _norm(name, rows, K, dtype, out, residual):
    return dict(name=name, kind="norm", rows=rows, K=K, dtype=dtype, out=out, residual=residual)


def _product(name, batch, M, K, dtype, bias, act):
    return dict(name=name, kind="product", batch=batch, M=M, K=K, dtype=dtype, bias=bias, act=act)


def _gated(name, batch, hidden, K, dtype):
    return dict(name=name, kind="product", batch=batch, M=2 * hidden, K=K, dtype=dtype, bias=False, act="gated")


def _block(name, batch, hidden, K, dtype):
    return dict(name=name, kind="block", batch=batch, M=2 * hidden, K=K, dtype=dtype, bias=False, act="gated")


def listed():
    return [
        # activations whose rows end inside a block and start at odd addresses
        _quantise("quantise-257x9219-f16", 257, 9219, "f16", 1),
        # the largest weight matrix of the benchmark configurations (VGG-16 fc6), as it is converted when a model is loaded
        _quantise("quantise-4096x25088-f32-w", 4096, 25088, "f32", 128),
        # one new token between two blocks
        _norm("norm-1x4096-bf16-f8", 1, 4096, "bf16", "f8", True),
        # a long prompt
        _norm("norm-16384x4096-bf16-f8", 16384, 4096, "bf16", "f8", True),
        # one request through AlexNet's fc6: reading the weights is the cost
        _product("product-b1-4096x9216", 1, 4096, 9216, "f32", True, "relu"),
        # a ragged batch through AlexNet's fc8
        _product("product-b37-1000x4096-bf16", 37, 1000, 4096, "bf16", True, "none"),
        # the headline batch through fc6
        _product("product-b256-4096x9216", 256, 4096, 9216, "f32", True, "relu"),
        # a long prompt, or a night's batch, through the largest layer
        _product("product-b4096-4096x25088-bf16", 4096, 4096, 25088, "bf16", False, "none"),
        # eight new tokens through both projections of a feed-forward block
        _gated("gated-b8-4096x4096-bf16", 8, 4096, 4096, "bf16"),
        # a few hundred tokens of ragged sizes
        _gated("gated-b333-2900x1100-f16", 333, 2900, 1100, "f16"),
        # the whole block for a few tokens, ragged sizes, and for a long prompt's
        _block("block-b19-2900x1100-bf16", 19, 2900, 1100, "bf16"),
        _block("block-b4096-9216x4096-bf16", 4096, 9216, 4096, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantise", "norm", "product", "gated", "block"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "quantise":
        K = _log(rng, 33, 25088)
        return dict(kind=kind, rows=_log(rng, 1, max(1, MOST_VALUES // K)), K=K, dtype=dtype, block_rows=rng.choice([1, 128]))
    if kind == "norm":
        K = _log(rng, 64, 16384)
        return dict(kind=kind, rows=_log(rng, 1, MOST_NORM // K), K=K, dtype=dtype, out=rng.choice([dtype, "f8"]), residual=rng.random() < 0.5)
    if kind == "product":
        M, K = _log(rng, 100, 4096), _log(rng, 100, 25088)
        return dict(kind=kind, batch=_log(rng, 1, 4096), M=M, K=K, dtype=dtype, bias=rng.random() < 0.5, act=rng.choice(["none", "relu"]))
    hidden, K = _log(rng, 100, 9216), _log(rng, 100, 9216)
    batch = _log(rng, 1, min(4096, int(MOST_FLOPS / (6.0 * hidden * K))))
    if kind == "block":
        return dict(kind=kind, batch=batch, M=2 * hidden, K=K, dtype=rng.choice(["bf16", "f16"]), bias=False, act="gated")
    return dict(kind="product", batch=batch, M=2 * hidden, K=K, dtype=dtype, bias=rng.random() < 0.3, act="gated")


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _activations(shape, dtype, gen):
    """What a layer reads: normal values whose size differs from row to row, as from token to token, and a few channels far larger than the rest."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), device="cuda", generator=gen))
    x *= 1.0 + 15.0 * (torch.rand(shape[-1], device="cuda", generator=gen) < 0.005)
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case=case)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "quantise":
        shape = (case["rows"], case["K"])
        if case["block_rows"] == 128:                              # weights: channels of different sizes
            state["X"] = (0.02 * torch.randn(shape, device="cuda", generator=gen) * torch.exp(0.5 * torch.randn((shape[0], 1), device="cuda", generator=gen))).to(dtype)
        else:
            state["X"] = _activations(shape, dtype, gen)
        return state
    if kind == "norm":
        state["X"] = _activations((case["rows"], case["K"]), dtype, gen)
        state["residual"] = (2.0 * _activations((case["rows"], case["K"]), torch.float32, gen)).to(dtype) if case["residual"] else None
        state["gain"] = (1.0 + 0.3 * torch.randn(case["K"], device="cuda", generator=gen)).to(dtype)
        return state
    # a matrix as a stored model has it, 8-bit values and scales; of a gated product the gates' and below it the values'
    halves = 2 if case["act"] == "gated" else 1
    rows, K = case["M"] // halves, case["K"]

    def matrix(M, K):
        return _to_blocks(torch.randn((M, K), device="cuda", generator=gen) * torch.exp(0.3 * torch.randn((M, 1), device="cuda", generator=gen)) * K ** -0.5, 128)

    parts = [matrix(rows, K) for _ in range(halves)]
    state["values"], state["scales"] = torch.cat([v for v, _ in parts]), torch.cat([s for _, s in parts])
    if kind == "block":
        state["down"] = matrix(K, rows)
    state["X"] = _activations((case["batch"], K), dtype, gen)
    state["bias"] = 0.1 * torch.randn(case["M"], device="cuda", generator=gen) if case["bias"] else None
    return state


# --------------------------------------------------------------------------- #
# the plain forms
# --------------------------------------------------------------------------- #
def _to_blocks(X, block_rows):
    """-> values (rows, whole blocks) in 8 bits and scales (row blocks, whole fours of blocks): the scale is the block's largest magnitude / 448, at least
    2^-126, a value the nearest 8-bit one of it times 448 / that magnitude.  What pads a row is zero."""
    rows, K = X.shape
    kb, tall = -(-K // BLOCK), -(-rows // block_rows)
    x = torch.nn.functional.pad(X.float(), (0, kb * BLOCK - K, 0, tall * block_rows - rows)).view(tall, block_rows, kb, BLOCK)
    top = x.abs().amax((1, 3))
    largest = torch.full_like(top, LARGEST)                        # (divided by, or dividing, a plain number is a product with a rounded reciprocal)
    scale = (top / largest).clamp_min(LEAST)
    inverse = torch.where(top < LARGEST * LEAST, 1 / LEAST, largest / top.clamp_min(LEAST))
    values = (x * inverse[:, None, :, None]).to(torch.float8_e4m3fn).view(tall * block_rows, kb * BLOCK)[:rows]
    return values.contiguous(), torch.nn.functional.pad(scale, (0, -kb % 4))


def _values(values, scales, K, block_rows):
    """What the blocks stand for, in 32 bits."""
    rows, kb = values.shape[0], values.shape[1] // BLOCK
    s = scales[:, :kb].repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)
    return (values.float() * s)[:, :K]


def _quantised(values, scales, K):
    return {"values": values[:, :K], "scales": scales[:, :-(-K // BLOCK)]}


def _plain_norm(s, case):
    x, total = s["X"].float(), None
    if s["residual"] is not None:
        total = (x + s["residual"].float()).to(s["X"].dtype)
        x = total.float()
    y = x / torch.sqrt((x * x).sum(1, keepdim=True) / case["K"] + EPS) * s["gain"].float()
    out = _quantised(*_to_blocks(y, 1), case["K"]) if case["out"] == "f8" else {"Y": y.to(s["X"].dtype)}
    return out if total is None else {**out, "sum": total}


def _plain_product(s, case):
    K, H = case["K"], case["M"] // 2
    x = _values(*_to_blocks(s["X"], 1), K, 1)
    if case["act"] == "gated":
        w = torch.cat([_values(v, t, K, 128) for v, t in zip(s["values"].split(H), s["scales"].chunk(2))])
    else:
        w = _values(s["values"], s["scales"], K, 128)
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["act"] == "gated":
        y = y[:, :H] / (1 + torch.exp(-y[:, :H])) * y[:, H:]
    elif case["act"] == "relu":
        y = torch.relu(y)
    if case["kind"] == "block":
        y = _values(*_to_blocks(y, 1), H, 1) @ _values(*s["down"], H, 128).t()
    return y.to(s["X"].dtype)


def run(state):
    case, X = state["case"], state["X"]
    kind = case["kind"]
    if own:
        import paper_1711_00244_amd as cl
        if kind == "quantise":
            q = cl.f8_quantize(X, block_rows=case["block_rows"])
            return _quantised(q.values, q.scales, q.K)
        if kind == "norm":
            y = cl.rms_norm(X, state["gain"], EPS, residual=state["residual"], dtype=DTYPES[case["out"]])
            y, total = y if case["residual"] else (y, None)
            out = _quantised(y.values, y.scales, y.K) if case["out"] == "f8" else {"Y": y}
            return out if total is None else {**out, "sum": total}
        W = cl.F8Tensor(state["values"], state["scales"], case["K"], block_rows=128, gated=case["act"] == "gated")
        if kind == "block":
            hidden = cl.f8_fc_forward(W, X, act="gated", dtype=torch.float8_e4m3fn)
            return cl.f8_fc_forward(cl.F8Tensor(*state["down"], case["M"] // 2, block_rows=128), hidden, dtype=X.dtype)
        return cl.f8_fc_forward(W, X, state["bias"], act=case["act"])
    if kind == "quantise":
        return _quantised(*_to_blocks(X, case["block_rows"]), case["K"])
    if kind == "norm":
        return _plain_norm(state, case)
    return _plain_product(state, case)


# --------------------------------------------------------------------------- #
# what a pass cannot do without
# --------------------------------------------------------------------------- #
def _bytes(rows, K, dtype, block_rows=1):
    return rows * K * SIZE[dtype] + (4 * -(-rows // block_rows) * -(-K // BLOCK) if dtype == "f8" else 0)


def work(case):
    kind, K = case["kind"], case["K"]
    if kind == "quantise":
        rows = case["rows"]
        return dict(bytes=_bytes(rows, K, case["dtype"]) + _bytes(rows, K, "f8", case["block_rows"]), flops=2 * rows * K)
    if kind == "norm":
        rows, dtype = case["rows"], case["dtype"]
        return dict(bytes=(3 if case["residual"] else 1) * _bytes(rows, K, dtype) + K * SIZE[dtype] + _bytes(rows, K, case["out"]), flops=6 * rows * K)
    B, M = case["batch"], case["M"]
    width = M // 2 if case["act"] == "gated" else M
    if kind == "block":
        return dict(bytes=_bytes(M, K, "f8", 128) + _bytes(K, width, "f8", 128) + 2 * _bytes(B, K, case["dtype"]), flops=2 * B * M * K + 2 * B * K * width)
    return dict(bytes=_bytes(M, K, "f8", 128) + _bytes(B, K, case["dtype"]) + _bytes(B, width, case["dtype"]) + (4 * M if case["bias"] else 0), flops=2 * B * M * K)


# --------------------------------------------------------------------------- #
# the definition in 64 bits
# --------------------------------------------------------------------------- #
def _blocks64(X, block_rows):
    """The values of X in blocks, not multiplied by their scales, and the scales.  The scale and the reciprocal that values are multiplied by are 32-bit
    numbers, as the operator has them, and so is the product; 8-bit steps are 2^-9 below 2^-6 and an eighth of the binade above."""
    rows, K = X.shape
    x = X.double()
    scale = torch.empty((-(-rows // block_rows), -(-K // 128)), dtype=torch.float64, device=X.device)
    codes = torch.empty((rows, K), dtype=torch.float64, device=X.device)
    for b in range(scale.shape[1]):
        part = x[:, 128 * b:128 * b + 128]
        top = torch.nn.functional.pad(part.abs().amax(1), (0, -rows % block_rows)).view(-1, block_rows).amax(1)
        most = torch.full_like(top, 448)
        scale[:, b] = (top / most).float().double().clamp_min(2.0 ** -126)
        by = torch.where(top < 448 * 2.0 ** -126, 2.0 ** 126, most / top.clamp_min(2.0 ** -126)).float().double()
        v = (part * by.repeat_interleave(block_rows)[:rows, None]).float().double()
        step = torch.exp2(torch.log2(v.abs().clamp_min(2.0 ** -6)).floor() - 3)
        step = torch.where(v.abs() >= 16 * step, 2 * step, step)     # (a logarithm that came out below its whole number)
        codes[:, 128 * b:128 * b + 128] = torch.round(v / step) * step
    return codes, scale


def _wide64(codes, scale, block_rows):
    rows, K = codes.shape
    return codes * scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :K]


def _stored64(values, scales, K):
    kb = values.shape[1] // 128
    return _wide64(values.double()[:, :K], scales.double()[:, :kb], 128)


def exact(case, seed):
    s = prepare(case, seed)
    kind, X, K = case["kind"], s["X"], case["K"]
    if kind == "quantise":
        codes, scale = _blocks64(X, case["block_rows"])
        return {"values": codes, "scales": scale}
    if kind == "norm":
        x, total = X.double(), None
        if s["residual"] is not None:
            total = (x + s["residual"].double()).to(X.dtype)
            x = total.double()
        y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * s["gain"].double()
        out = {"Y": y}
        if case["out"] == "f8":
            codes, scale = _blocks64(y, 1)
            out = {"values": codes, "scales": scale}
        return out if total is None else {**out, "sum": total.double()}
    x = _wide64(*_blocks64(X, 1), 1)
    if case["act"] == "gated":
        H, tall = case["M"] // 2, s["scales"].shape[0] // 2
        parts = [(s["values"][:H], s["scales"][:tall]), (s["values"][H:], s["scales"][tall:])]
    else:
        parts = [(s["values"], s["scales"])]
    y = torch.cat([torch.cat([x @ _stored64(v[r:r + 1024], t[r // 128:r // 128 + 8], K).t() for r in range(0, len(v), 1024)], 1) for v, t in parts], 1)
    if s["bias"] is not None:
        y = y + s["bias"].double()
    if case["act"] == "gated":
        y = y[:, :H] * torch.sigmoid(y[:, :H]) * y[:, H:]
    elif case["act"] == "relu":
        y = y.clamp_min(0)
    if kind == "block":
        x = _wide64(*_blocks64(y, 1), 1)
        v, t = s["down"]
        y = torch.cat([x @ _stored64(v[r:r + 1024], t[r // 128:r // 128 + 8], H).t() for r in range(0, K, 1024)], 1)
    return y
