"""Plain forms of the 8-bit operators in numpy (fp64, and fp32 where the definition rounds to it), and the error gates of their results.

Gates.  Within a block products of two 8-bit values are exact, and of the 128 additions in fp32, in any order, each is off by at most one unit in the last place (a
matrix unit may truncate where other arithmetic rounds); outputs in bf16 and fp16 come from the 8-bit matrix instruction, which cuts seven of each run of
eight products off at 2^-13 of the largest (product(), eights).  A block's sum is multiplied by a rounded product of two scales and
added to K / 128 others with one rounding each, a bias, and partial sums: all of it within (K + 8) 2^-23 of the terms' absolute sum.  Rounding to the
output's type adds half a step: 2^-24, 2^-8 (bf16), 2^-11 (fp16; 2^-25 below its normal numbers), and of 8 bits 2^-4 of the value or, below their normal
numbers, 2^-10 of the scale."""
import numpy as np
import torch

import mx_ref
from mx_ref import DTYPES  # noqa: F401

F8 = torch.float8_e4m3fn
LEAST = np.float32(2.0 ** -126)


def blocks(K):
    return -(-K // 128)


def e4m3(v):
    """The nearest 8-bit value of each of v (|v| below 464), ties to even, as float64."""
    v = np.asarray(v, np.float64)
    e = np.maximum(np.frexp(np.where(v == 0, 1.0, v))[1] - 1, -6)
    step = 2.0 ** (e - 3.0)
    return np.copysign(np.minimum(np.round(np.abs(v) / step) * step, 448.0), v)


def quantise(x, block_rows=1):
    """x (rows, K), values of fp32 or fewer bits -> 8-bit values as float64 (rows, blocks * 128), scales float32 (row blocks, blocks)."""
    x = np.asarray(x, np.float32)
    rows, K = x.shape
    kb, tall = blocks(K), -(-rows // block_rows)
    p = np.zeros((tall * block_rows, kb * 128), np.float32)
    p[:rows, :K] = x
    p = p.reshape(tall, block_rows, kb, 128)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(p).all(axis=(1, 3))
        top = np.where(bad, np.float32(1), np.abs(p).max(axis=(1, 3)))
        low = top < np.float32(448) * LEAST
        scale = np.maximum(top / np.float32(448), LEAST)
        by = np.where(low, 1 / LEAST, np.float32(448) / np.where(low, np.float32(1), top))
        v = e4m3(np.where(bad[:, None, :, None], np.float32(0), p * by[:, None, :, None].astype(np.float32)))
    v = np.where(bad[:, None, :, None], 0.0, v)
    return v.reshape(tall * block_rows, kb * 128)[:rows], np.where(bad, np.float32(np.nan), scale).astype(np.float32)


def values(codes, scales, K, block_rows=1):
    """What 8-bit values (rows, blocks * 128) and scales (row blocks, at least blocks) stand for, (rows, K) float64."""
    rows, kb = codes.shape[0], blocks(K)
    s = np.repeat(np.repeat(scales[:, :kb].astype(np.float64), block_rows, 0)[:rows], 128, 1)
    return (codes.astype(np.float64) * s)[:, :K]


def stored(q):
    """(8-bit values as float64, scales) of an F8Tensor."""
    return q.values.view(torch.uint8).cpu().view(F8).double().numpy(), q.scales.cpu().numpy()


def stand_for(q):
    """What an F8Tensor stands for, float64; of a gated matrix each half with its own scales."""
    v, s = stored(q)
    if q.gated:
        h, t = len(v) // 2, len(s) // 2
        return np.concatenate([values(v[:h], s[:t], q.K, 128), values(v[h:], s[t:], q.K, 128)])
    return values(v, s, q.K, q.block_rows)


def quantised(x):
    """The values that rows of x are rounded to."""
    x = np.asarray(x)
    return values(*quantise(x), x.shape[1])


def eights(xq, wq):
    """The sum over runs of eight k of the largest product, (rows of xq, rows of wq)."""
    K = xq.shape[1]
    x, w = (torch.from_numpy(np.pad(np.abs(v), ((0, 0), (0, -K % 8)))).float() for v in (xq, wq))
    total = torch.zeros((len(xq), len(wq)))
    for k in range(0, K, 8):
        most = x[:, k, None] * w[:, k]
        for i in range(1, 8):
            most = torch.maximum(most, x[:, k + i, None] * w[:, k + i])
        total += most
    return total.double().numpy() * (1 + K * 2.0 ** -23)


def product(xq, wq, bias, act, most=None):
    """-> (result, bound of its error before the rounding to the output's type); gated: rows 0 .. H - 1 of wq gates, the others values.  most: eights() of
    the operands, for outputs in bf16 and fp16."""
    pre, size = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    if bias is not None:
        pre, size = pre + bias, size + np.abs(bias)
    err = (wq.shape[1] + 8) * 2.0 ** -23 * size
    if most is not None:
        err = err + 7 * 2.0 ** -13 * most
    if act == "gated":
        H = wq.shape[0] // 2
        g, u, eg, eu = pre[:, :H], pre[:, H:], err[:, :H], err[:, H:]
        silu = g / (1 + np.exp(-g))
        out = silu * u
        return out, 1.1 * np.abs(u) * eg + (np.abs(silu) + 1.1 * eg) * eu + np.abs(out) * (8 + np.abs(g)) * 2.0 ** -23
    return (np.where(pre < 0, 0.0, pre) if act == "relu" else pre), err


def norm(h, gain, eps):
    """h (rows, K) float64 -> (result, bound).  A lane adds up to 64 squares, and one for each 1024 of a row beyond what lanes hold; then lanes (6) and
    wavefronts (16); the root halves the relative error; mean, eps, root, quotient and two products round once each."""
    K = h.shape[1]
    y = h / np.sqrt((h * h).sum(1, keepdims=True) / K + eps)
    if gain is not None:
        y = y * gain
    return y, np.abs(y) * (0.5 * (64 + 8 + K / 1024 + 22 + 2) + 5) * 2.0 ** -24


def assert_within(Y, want, err, what=None):
    """mx_ref's, but for results that fp16 rounds to Inf: those of 65520 and more, halfway from its largest number to the next step."""
    if Y.dtype == torch.float16:
        y = Y.double().cpu().numpy()
        over = np.isinf(y) & (np.sign(y) == np.sign(want)) & (np.abs(want) + err >= 65520)
        Y, want = torch.where(torch.from_numpy(over).to(Y.device), torch.zeros_like(Y), Y), np.where(over, 0.0, want)
    mx_ref.assert_within(Y, want, err, what)


def assert_f8_within(q, want, err, what=None):
    """An F8Tensor against the fp64 result that it holds in 8 bits: its scales, and its values within half a step."""
    v, s = stored(q)
    rows, K = want.shape
    kb = blocks(K)
    assert q.shape == (rows, K) and v.shape == (rows, kb * 128), what
    assert (v[:, K:] == 0).all() and (s[:, kb:] == 0).all(), what
    p, e = np.zeros((rows, kb * 128)), np.zeros((rows, kb * 128))
    p[:, :K], e[:, :K] = want, err
    p, e = p.reshape(rows, kb, 128), e.reshape(rows, kb, 128)
    bad = ~np.isfinite(p).all(2)
    assert np.array_equal(np.isnan(s[:, :kb]), bad), what
    if bad.any():
        p, e = np.where(bad[:, :, None], 0.0, p), np.where(bad[:, :, None], 0.0, e)
    top = np.abs(p).max(2)
    scale = np.where(bad, 0.0, s[:, :kb].astype(np.float64))
    lo, hi = np.maximum(np.max(np.abs(p) - e, axis=2) / 448, float(LEAST)), np.maximum((np.max(np.abs(p) + e, axis=2)) / 448, float(LEAST))
    assert ((scale >= lo * (1 - 2.0 ** -23)) & (scale <= hi * (1 + 2.0 ** -23)) | bad).all(), what
    got = v.reshape(rows, kb, 128) * scale[:, :, None]
    # (half a step of the value; what is multiplied to come within the range is rounded three times, 2^-24 each)
    bound = (np.abs(p) + e) * (2.0 ** -4 + 2.0 ** -21) + e + scale[:, :, None] * 2.0 ** -10
    off = np.abs(got - p)
    assert (off <= bound).all(), (what, float((off / np.maximum(bound, 1e-300)).max()), float(top.max()))
