"""A layer of routed experts behind a compressed layer: the router is a pruned, codebook-quantised, Huffman-coded layer of this library,
the experts are gated two-matrix networks in 4-bit blocks.  One call is

    logits = compressed_fc_forward(router, X)                       float32, (tokens, experts)
    chosen, weights = route_experts(logits, k, ...)
    lists = expert_lists(chosen, experts)                           once for both products; not where both are one launch without
    hidden = mx_experts_forward(up, X, chosen, act="gated")         a row per pair
    Y = mx_experts_forward(down, hidden, chosen, weights, ...)      a row per token

and, where there is a shared expert, mx_fc_forward of its two matrices on X, quantised once for the shared expert and the routed ones.  A shared expert, which every
token goes through, may be in 8 bits instead (f8_fc_forward).
Host-side control only: the work is in the library's kernels, on the caller's current stream, and nothing is read back, so that a call can be
recorded in a graph.

    python -m paper_1711_00244_amd.experts                          # 1, 64 and 4096 tokens; one JSON line each
"""
from __future__ import annotations

import argparse
import json

import numpy as np

from . import binding as cl
from . import feed_forward
from . import workloads as wl

SHARED_QUANTISE_TOKENS = 64      # below, each product quantises X itself: the few rows of those that are one launch, in that launch


class ExpertLayer:
    """router: a compressed layer of (experts, width); up: MxTensor (experts, 2 hidden, width), rows 2 i and 2 i + 1 gate and value of hidden
    unit i; down: MxTensor (experts, width, hidden); shared: None or (MxTensor (2 h, width), MxTensor (width, h)), or two F8Tensors of these shapes, the
    first as f8_gated makes it.  routing: keyword arguments of route_experts."""

    def __init__(self, router: cl.Layer, up: cl.MxTensor, down: cl.MxTensor, k: int, shared=None, **routing):
        experts, two_hidden, width = up.shape
        if (router.M, router.K) != (experts, width):
            raise ValueError(f"the router must be {experts} x {width}, is {router.M} x {router.K}")
        if two_hidden % 2 or down.shape != (experts, width, two_hidden // 2):
            raise ValueError(f"up {up.shape} and down {down.shape} are not the matrices of gated experts")
        if shared is not None:
            first, second = shared
            if isinstance(first, cl.F8Tensor) or isinstance(second, cl.F8Tensor):
                feed_forward.check_gated(first, second)
            if len(first.shape) != 2 or first.K != width or first.shape[0] % 2 or second.shape != (width, first.shape[0] // 2):
                raise ValueError(f"{first.shape} and {second.shape} are not the matrices of a gated expert of width {width}")
        self.router, self.up, self.down, self.k, self.shared, self.routing = router, up, down, k, shared, routing
        self.experts, self.width = experts, width

    def route(self, X):
        """-> experts (tokens, k), weights (tokens, k); X float32."""
        return cl.route_experts(cl.compressed_fc_forward(self.router, X), self.k, **self.routing)

    def forward(self, X):
        """X (tokens, width) float32 -> (tokens, width) float32."""
        if X.shape[0] == 0:
            return X.new_empty((0, self.width))              # (a compressed layer takes no empty batch)
        experts, weights = self.route(X)
        eight = self.shared is not None and isinstance(self.shared[0], cl.F8Tensor)
        x = cl.mx_quantize(X) if self.shared is not None and not eight and X.shape[0] >= SHARED_QUANTISE_TOKENS else X
        # (of the default layer up to 15 tokens.  One token, calls recorded in a graph: 29 us, with lists 37; called one by one 63, with lists 80)
        one_launch = ("few" == cl.mx_experts_resolved_form(self.up, X.shape[0], self.k, None if x is not X else X.dtype, weighted=False)
                      == cl.mx_experts_resolved_form(self.down, X.shape[0], self.k, X.dtype, x_per_pair=True))
        lists = None if one_launch else cl.expert_lists(experts, self.experts)
        hidden = cl.mx_experts_forward(self.up, x, experts, act="gated", lists=lists, dtype=X.dtype)
        Y = cl.mx_experts_forward(self.down, hidden, experts, weights, x_per_pair=True, lists=lists)
        if eight:
            Y += feed_forward.gated_product(*self.shared, X, X.dtype)
        elif self.shared is not None:
            first, second = self.shared
            Y += cl.mx_fc_forward(second, cl.mx_fc_forward(first, x, act="gated", dtype=X.dtype))
        return Y


def synthetic(experts=64, width=1024, hidden=512, k=6, shared=True, density=0.25, seed=0, **routing) -> ExpertLayer:
    """Seeded weights: a pruned router compressed at 5-bit codes, experts drawn on the device and quantised."""
    import torch
    W = wl.pruned_weights(experts, width, density, (1.0 / (density * width)) ** 0.5, seed)
    router = cl.compress_layer(W, 5, 5, min(128, experts), 128, upload=True)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape):
        return cl.mx_quantize(torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * shape[-1] ** -0.5)

    both = (draw(2 * hidden, width), draw(width, hidden)) if shared else None
    return ExpertLayer(router, draw(experts, 2 * hidden, width), draw(experts, width, hidden), k, both, **routing)


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--k", type=int, default=6)
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 64, 4096])
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    layer = synthetic(args.experts, args.width, args.hidden, args.k, score="sigmoid", groups=8 if args.experts % 8 == 0 else 1)
    for tokens in args.tokens:
        X = torch.from_numpy(np.random.default_rng(tokens).standard_normal((tokens, args.width), dtype=np.float32)).cuda()
        for _ in range(3):
            layer.forward(X)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        begin.record()
        for _ in range(args.steps):
            layer.forward(X)
        end.record()
        torch.cuda.synchronize()
        print(json.dumps({"tokens": tokens, "experts": args.experts, "k": args.k, "width": args.width, "hidden": args.hidden,
                          "ms": round(begin.elapsed_time(end) / args.steps, 4)}), flush=True)


if __name__ == "__main__":
    main()
