"""A gated feed-forward block in 8 bits: a root-mean-square norm that adds the residual, both projections with their activation and product, and the
second matrix.  One call is three launches and, for a few tokens, one or two small ones between them:

    h, total = rms_norm(X, gain, residual=residual, dtype=float8_e4m3fn)       8 bits with a scale for each 128 of a row
    hidden = f8_fc_forward(up, h, act="gated", dtype=float8_e4m3fn)            the same
    Y = f8_fc_forward(down, hidden, dtype=X.dtype)

Host-side control only: the work is in the library's kernels, on the caller's current stream, and nothing is read back, so that a call can be
recorded in a graph.

    python -m paper_1711_00244_amd.feed_forward                     # 1, 64 and 4096 tokens; one JSON line each
"""
from __future__ import annotations

import argparse
import json

from . import binding as cl


class GatedLayer:
    """up: F8Tensor (2 hidden, width), gates and values as f8_gated makes it; down: F8Tensor (width, hidden) in blocks of 128 rows; gain: (width),
    float32 or of the tokens' type, or None."""

    def __init__(self, up: cl.F8Tensor, down: cl.F8Tensor, gain=None, eps: float = 1e-6):
        check_gated(up, down)
        if gain is not None and tuple(gain.shape) != (up.K,):
            raise ValueError(f"gain must be ({up.K},), is {tuple(gain.shape)}")
        self.up, self.down, self.gain, self.eps, self.width = up, down, gain, eps, up.K

    def forward(self, X, residual=None):
        """X (tokens, width), float32, bfloat16 or float16 -> (tokens, width); with a residual of that shape (Y, X + residual)."""
        import torch
        h = cl.rms_norm(X, self.gain, self.eps, residual=residual, dtype=torch.float8_e4m3fn)
        h, total = h if residual is not None else (h, None)
        Y = gated_product(self.up, self.down, h, X.dtype)
        return Y if total is None else (Y, total)


def check_gated(up, down):
    """up and down are the matrices of a gated block, as f8_fc_forward takes them."""
    if not (isinstance(up, cl.F8Tensor) and isinstance(down, cl.F8Tensor)):
        raise ValueError(f"the matrices of a gated block must be two F8Tensors, are {type(up).__name__} and {type(down).__name__}")
    if up.block_rows != 128 or down.block_rows != 128 or down.gated or len(up.shape) != 2 or up.shape[0] % 2 or tuple(down.shape) != (up.K, up.shape[0] // 2):
        raise ValueError(f"{up.shape} and {down.shape} are not the matrices of a gated block in blocks of 128 rows")
    if not up.gated and up.shape[0] % 256:
        raise ValueError(f"{up.shape}: gates and values in halves that are no multiple of 128 rows have to be put together by f8_gated")


def gated_product(up, down, X, dtype):
    """Both matrices of a gated block on X (numbers, or an F8Tensor), what is between them in 8 bits -> dtype."""
    import torch
    return cl.f8_fc_forward(down, cl.f8_fc_forward(up, X, act="gated", dtype=torch.float8_e4m3fn), dtype=dtype)


def synthetic(width=4096, hidden=9216, seed=0) -> GatedLayer:
    """Seeded weights, drawn on the device and quantised."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(rows, K):
        return cl.f8_quantize(torch.randn((rows, K), generator=g, device="cuda", dtype=torch.float32) * K ** -0.5, block_rows=128)

    return GatedLayer(cl.f8_gated(draw(hidden, width), draw(hidden, width)), draw(width, hidden), 1 + 0.1 * torch.randn(width, generator=g, device="cuda"))


def main():
    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=9216)
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 64, 4096])
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    layer = synthetic(args.width, args.hidden)
    for tokens in args.tokens:
        g = torch.Generator(device="cuda").manual_seed(tokens)
        X, residual = (torch.randn((tokens, args.width), generator=g, device="cuda").bfloat16() for _ in range(2))
        for _ in range(3):
            layer.forward(X, residual)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        begin.record()
        for _ in range(args.steps):
            layer.forward(X, residual)
        end.record()
        torch.cuda.synchronize()
        print(json.dumps({"tokens": tokens, "width": args.width, "hidden": args.hidden, "ms": round(begin.elapsed_time(end) / args.steps, 4)}), flush=True)


if __name__ == "__main__":
    main()
