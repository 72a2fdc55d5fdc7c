"""Plain 64-bit implementations of the operators for networks that the caller runs itself (selection from logits, reordering of states, the
paged cache and the attention over it), and inputs for them.  numpy, one row at a time; nothing here is shared with the library."""
from __future__ import annotations

import math

import numpy as np

HALF_STEP = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}


def torch_type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


# ---------------------------------------------------------------- selection
def select(logits, scores, done=None, eos=-1):
    """(scores, parents, tokens, done) of logits [B, beam, V] in float64."""
    B, K, V = logits.shape
    out = np.full((B, K), -np.inf), np.full((B, K), -1, np.int32), np.full((B, K), -3, np.int32), np.zeros((B, K), bool)
    for b in range(B):
        keys = np.full((K, V), -np.inf)
        for k in range(K):
            if done is not None and done[b, k]:
                keys[k, eos] = scores[b, k]
                continue
            x = logits[b, k]
            if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
                continue
            top = x.max()
            keys[k] = scores[b, k] + (x - (top + math.log(np.exp(x - top).sum())))
        flat = keys.reshape(-1)
        flat = np.where(np.isnan(flat), -np.inf, flat)
        # of equal keys the smaller hypothesis, the larger logit (keys of two may round to one), the smaller token
        order = np.lexsort((np.arange(K * V), -np.nan_to_num(logits[b].reshape(-1)), np.repeat(np.arange(K), V), -flat))[:K]
        for r, at in enumerate(order):
            if flat[at] > -np.inf:
                out[0][b, r], out[1][b, r], out[2][b, r], out[3][b, r] = flat[at], at // V, at % V, at % V == eos
    return out


def select_margin(logits, scores, done=None, eos=-1):
    """Smallest gap between neighbours among the first beam + 1 keys that are not equal bit for bit."""
    B, K, V = logits.shape
    least = np.inf
    for b in range(B):
        keys = []
        for k in range(K):
            if done is not None and done[b, k]:
                keys.append(np.array([scores[b, k]]))
                continue
            x = logits[b, k]
            if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
                continue
            top = x.max()
            keys.append(scores[b, k] + (x - (top + math.log(np.exp(x - top).sum()))))
        if not keys:
            continue
        keys = np.concatenate(keys)
        keys = -np.sort(-keys[keys > -np.inf])[:K + 1]
        gaps = -np.diff(keys)
        gaps = gaps[gaps > 0]
        least = min(least, gaps.min(initial=np.inf))
    return least


# ---------------------------------------------------------------- the cache's formats
def quantise(x, fmt):
    """(y, exponent byte) of one row in float64."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros_like(x), 255
    most = np.abs(x).max()
    if most == 0:
        return np.zeros_like(x), 127
    mant, e = math.frexp(most)  # most = mant 2^e, mant in [1/2, 1)
    if fmt == "f16":
        s, digits, least = e - 15, 11, -14
    else:
        s, digits, least = (e - 8 if mant > 0.875 else e - 9), 4, -6
    s = max(s, -126)
    y = np.ldexp(x, -s)
    unit = np.ldexp(1.0, np.maximum(np.frexp(y)[1] - 1, least) - (digits - 1))
    return np.rint(y / unit) * unit, s + 127


def stands_for(y, e):
    return np.asarray(y, np.float64) * (math.nan if e == 255 else 2.0 ** (e - 127))


# ---------------------------------------------------------------- attention
def path_of(parents, i):
    """Node i and its ancestors, or None for padding."""
    path = []
    while True:
        if not -1 <= parents[i] < i:
            return None
        path.append(i)
        if parents[i] == -1:
            return path
        i = parents[i]


def attend(q, k, v, lens, parents, scale):
    """q [B, n, q_heads, dim]; k, v [B][tokens][heads][dim] (float64, NaN rows where nothing was written); parents [B][tree].  float64 [B, n, q_heads, dim]
    and, for the tolerances, sum p |v| and the largest |x| of each query."""
    B, n, Hq, D = q.shape
    out, size, far = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        tree = len(parents[b])
        group = Hq // k[b].shape[1]
        for i in range(n):
            path = path_of(parents[b], tree - n + i)
            if path is None:
                continue
            at = np.array([t for t in list(range(max(int(lens[b]), 0))) + [max(int(lens[b]), 0) + j for j in path[::-1]] if t < len(k[b])], int)
            if not len(at):
                continue
            for h in range(Hq):
                kk, vv = k[b][at, h // group], v[b][at, h // group]
                x = scale * (kk @ q[b, i, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                out[b, i, h] = p @ vv
                size[b, i, h] = p @ np.abs(vv)
                far[b, i, h] = scale * (np.abs(kk) @ np.abs(q[b, i, h])).max()
    return out, size, far
