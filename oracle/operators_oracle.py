"""CPU statements of the 4-bit product and of the logits step (test infrastructure; share no code with the library)."""
from __future__ import annotations

import numpy as np

NO_TOKEN = 0x7FFFFFFF


# ---- out = sum_g scale * sum_{k in g} (q - zero) x ------------------------------------------------------------
def q4_unpack(Wq):
    """[N, K / 2] bytes -> [N, K] integers, low four bits first."""
    Wq = np.asarray(Wq, np.uint8)
    q = np.empty((Wq.shape[0], 2 * Wq.shape[1]), np.int64)
    q[:, 0::2] = Wq & 15
    q[:, 1::2] = Wq >> 4
    return q


def q4_linear(Wq, scales, zeros, x):
    """(out [M, N], size [M, N]): the product in float64 and the same sum over absolute values."""
    q = q4_unpack(Wq).astype(np.float64)
    group = q.shape[1] // scales.shape[1]
    z = 8.0 if zeros is None else np.repeat(np.asarray(zeros, np.float64), group, axis=1)
    W = (q - z) * np.repeat(np.asarray(scales, np.float64), group, axis=1)
    x = np.asarray(x, np.float64)
    return x @ W.T, np.abs(x) @ np.abs(W).T


# ---- penalties, biases, masks, candidates ----------------------------------------------------------------------
def logits_row(l, V, k, prompt=(), output=(), path=(), rep=None, freq=None, pres=None, bias=(), mask=None, nothing=False):
    """One row, step by step in float32.  bias: (token, value) pairs in list order; mask: words or None.
    Returns (processed float32 [V], ids [k], logprobs [k] float64, lse float64)."""
    v = np.array(l, np.float32)
    f32 = np.float32
    count = np.zeros(V, np.int64)
    seen = np.zeros(V, bool)
    for t in list(output) + list(path):
        if 0 <= t < V:
            count[t] += 1
    for t in prompt:
        if 0 <= t < V:
            seen[t] = True
    seen |= count > 0
    with np.errstate(all="ignore"):
        for t in np.nonzero(seen)[0]:
            if rep is not None:
                v[t] = v[t] / f32(rep) if v[t] > 0 else v[t] * f32(rep)
            if count[t]:
                if freq is not None:
                    v[t] = v[t] - f32(f32(freq) * f32(count[t]))
                if pres is not None:
                    v[t] = v[t] - f32(pres)
        last = {}
        for t, b in bias:
            last[int(t)] = b
        for t, b in last.items():
            if 0 <= t < V:
                v[t] = v[t] + f32(b)
    if nothing:
        v[:] = -np.inf
    elif mask is not None:
        bits = np.unpackbits(np.asarray(mask, np.uint32).view(np.uint8), bitorder="little")[:V].astype(bool)
        v[~bits] = -np.inf
    d = v.astype(np.float64)
    if np.any(np.isnan(d)) or np.any(np.isposinf(d)):
        lse = np.nan
    elif np.all(np.isneginf(d)):
        lse = -np.inf
    else:
        lse = d.max() + np.log(np.sum(np.exp(d - d.max())))
    order = [t for t in np.lexsort((np.arange(V), -np.where(np.isnan(d), -np.inf, d)))[:k] if d[t] > -np.inf]
    ids = np.full(k, NO_TOKEN, np.int64)
    lps = np.full(k, -np.inf)
    ids[:len(order)] = order
    with np.errstate(invalid="ignore"):
        lps[:len(order)] = d[order] - lse
    return v, ids, lps, lse
