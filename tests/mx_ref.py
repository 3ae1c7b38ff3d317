"""Plain fp64 forms of the microscaled 4-bit operators and of routed experts, and the error gates of their products.

Gates.  Products of two codes and their scales are exact; a sum of n of them in fp32, in any order, each addition off by at
most one unit in the last place (a matrix unit may truncate where other arithmetic rounds), is within (n + 4) 2^-23 of the
terms' absolute sum (+4: the bias, the additions of partial sums beyond n, the weighting).  Rounding to the output's type adds the
unit roundoff of its significand (24, 8, 11 bits): 2^-24, 2^-8 (bf16), 2^-11 (fp16) of the output, or half the smallest subnormal of fp16, 2^-25.  A gated
output is silu(g) u, whose derivatives are below 1.1 |u| and |silu(g)|; exp and the division add a few units more."""
import numpy as np
import torch

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def blocks(K):
    return -(-K // 128) * 4


def quantise(x):
    """x (rows, K) float64 -> codes (rows, blocks * 16) uint8, scales (rows, blocks) uint8."""
    rows, K = x.shape
    kb = blocks(K)
    p = np.zeros((rows, kb * 32))
    p[:, :K] = x
    p = p.reshape(rows, kb, 32)
    top = np.abs(p).max(axis=2, initial=0.0)
    bad = ~np.isfinite(p).all(axis=2)
    e = np.frexp(np.where(bad, 1.0, top))[1] - 1                 # floor(log2)
    s = np.clip(np.where(top > 0, e - 2, -127), -127, 127)
    a = np.abs(np.where(bad[:, :, None], 0.0, p)) * 2.0 ** -s[:, :, None].astype(np.float64)
    # nearest of the grid, ties to the even code
    d = np.abs(a[..., None] - GRID)
    near = d.min(axis=-1, keepdims=True)
    code = np.where((d == near) & (np.arange(8) % 2 == 0), 8 + np.arange(8), np.where(d == near, np.arange(8), -1)).max(axis=-1) % 8
    code = code + 8 * (np.signbit(p) & ~bad[:, :, None])
    code = code.astype(np.uint8).reshape(rows, -1, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, np.where(bad, 255, s + 127).astype(np.uint8)


def values(codes, scales, K):
    """(..., K) float64."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(s, 32, axis=-1))[..., :K]


def quantised(x):
    """The values that x is rounded to."""
    x = np.asarray(x, np.float64)
    return values(*quantise(x), x.shape[1])


def activate(v, act):
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    if act == "gated":
        g, u = v[..., 0::2], v[..., 1::2]
        return g / (1 + np.exp(-g)) * u
    return v


def product(xq, wq, bias, act):
    """-> (result, bound of its fp32 error before the rounding to the output's type)"""
    pre = xq @ wq.T
    size = np.abs(xq) @ np.abs(wq).T
    if bias is not None:
        pre, size = pre + bias, size + np.abs(bias)
    err = (wq.shape[1] + 4) * 2.0 ** -23 * size
    if act == "gated":
        g, u = pre[..., 0::2], pre[..., 1::2]
        silu = g / (1 + np.exp(-g))
        out = silu * u
        err = 1.1 * np.abs(u) * err[..., 0::2] + (np.abs(silu) + 1.1 * err[..., 0::2]) * err[..., 1::2] + np.abs(out) * (8 + np.abs(g)) * 2.0 ** -23
        return out, err
    return activate(pre, act), err


def experts(xq, wq, e, weights, bias, act, x_per_pair):
    """wq (E, M, K), e (T, k) -> (result, bound)"""
    T, k = e.shape
    E, M = wq.shape[:2]
    width = M // 2 if act == "gated" else M
    P, err = np.zeros((T * k, width)), np.zeros((T * k, width))
    for p, n in enumerate(e.reshape(-1)):
        if 0 <= n < E:
            P[p], err[p] = product(xq[p if x_per_pair else p // k][None], wq[n], None if bias is None else bias[n], act)
    if weights is None:
        return P, err
    w = np.asarray(weights, np.float64).reshape(T, k, 1)
    P, err = P.reshape(T, k, width), err.reshape(T, k, width)
    return (w * P).sum(1), (np.abs(w) * err).sum(1) + (k + 1) * 2.0 ** -23 * np.abs(w * P).sum(1)


def assert_within(Y, ref, err, what=None):
    """Y, a tensor, against the fp64 result within the bound of its arithmetic and its type's rounding."""
    dtype = Y.dtype
    Y = Y.double().cpu().numpy()
    assert Y.shape == ref.shape, (Y.shape, ref.shape, what)
    assert np.array_equal(np.isnan(Y), np.isnan(ref)), what
    bound = err + HALF_ULP[dtype] * (np.abs(ref) + err) + SMALLEST[dtype]
    off = np.abs(Y - ref)
    ok = (off <= bound) | np.isnan(ref)
    assert ok.all(), (what, float(off[~ok].max()), float((off[~ok] / bound[~ok]).max()), int((~ok).sum()))


def route(x, bias, k, score, groups, kept, group_score, renormalize, scale, lowest):
    """x (T, E) float64 -> (experts, weights, sure): sure where no two keys or group scores whose order decides something are apart by less than
    the rounding of fp32 arithmetic but not equal by their inputs."""
    T, E = x.shape
    size = E // groups
    out, w, sure = np.full((T, k), -1, np.int32), np.zeros((T, k)), np.ones(T, bool)

    def close(v, n):
        """v descending: whether the order of its first n and the next one may come out differently."""
        v = v[:n + 1]
        gap = v[:-1][np.isfinite(v[1:])] - v[1:][np.isfinite(v[1:])]
        return (gap <= 1e-6 * np.maximum(np.abs(v[1:][np.isfinite(v[1:])]), 1e-3)).any()

    for t in range(T):
        live = x[t] > lowest
        if not live.any():
            continue
        if score == "softmax":
            top = x[t][live].max()
            s = np.where(live, np.where(x[t] == top, 1.0, np.exp(np.where(live, x[t], -np.inf) - top) if np.isfinite(top) else 0.0), 0.0)
            s = s / s.sum()
        else:
            s = np.where(live, 1 / (1 + np.exp(-np.where(live, x[t], 0.0))), 0.0)
        biased = s if bias is None else s + bias
        live = live & ~np.isnan(biased) & (biased > -np.inf)
        key = np.where(live, x[t] if bias is None else biased, -np.inf)
        if groups > 1:
            of = []
            for g in range(groups):
                v = np.sort(biased[g * size:(g + 1) * size][live[g * size:(g + 1) * size]])[::-1]
                of.append(-np.inf if not len(v) else v[0] + v[1] if group_score == "top2" and len(v) > 1 else v[0])
            of = np.array(of)
            order = np.argsort(-of, kind="stable")
            if kept < groups and np.isfinite(of[order[kept]]) and close(of[order[kept - 1:kept + 1]], 1):
                sure[t] = False
            key = np.where(np.isin(np.arange(E) // size, order[:kept]), key, -np.inf)
        order = np.argsort(-key, kind="stable")
        first = order[:k + 1][key[order[:k + 1]] > -np.inf]
        # equal keys of equal inputs are in order whatever the arithmetic: only the first of a run counts
        run = np.array([i == 0 or x[t][first[i]] != x[t][first[i - 1]] or (bias is not None and bias[first[i]] != bias[first[i - 1]]) for i in range(len(first))], bool)
        if bias is not None and len(first) and close(key[first[run]], k):
            sure[t] = False
        first = first[:k]
        out[t, :len(first)] = first
        v = s[first]
        if renormalize:
            v = v / v.sum() if v.sum() > 0 else v * 0
        w[t, :len(first)] = v * scale
    return out, w, sure
