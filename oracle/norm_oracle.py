"""CPU float64 statement of the block norm and of its gradient (test infrastructure; shares no code with the library).

    b = w_post ? x / sqrt(mean(x^2) + eps) * w_post : x
    y = alpha * r + gate * b
    h = y / sqrt(mean(y^2) + eps) * w_pre

`gate` broadcasts: None, [H], [M, 1] or [M, H].  Next to every result the functions return the size of what was added up to
it (the same formula over absolute values): rounding errors of a float32 evaluation are small against that, not always
against the result itself.
"""
from __future__ import annotations

import numpy as np


def _rms(v, eps):
    return 1.0 / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps)


def forward(x, r, w_pre, eps, w_post=None, gate=None, alpha=1.0):
    x = np.asarray(x, np.float64)
    g = 1.0 if gate is None else np.asarray(gate, np.float64)
    b = x if w_post is None else x * _rms(x, eps) * w_post
    res = 0.0 if r is None else alpha * np.asarray(r, np.float64)
    y = res + g * b
    size_y = np.abs(res) + np.abs(g * b)
    if w_pre is None:
        return y, None, size_y, None
    ry = _rms(y, eps)
    h = y * ry * w_pre
    spread = np.sqrt(np.mean(size_y ** 2, axis=1, keepdims=True)) * ry       # how far y is smaller than its parts
    size_h = np.abs(w_pre) * ry * (size_y + np.abs(y) * (1.0 + spread))
    return y, h, size_y, size_h


def backward(x, r, w_pre, eps, dy, dh, w_post=None, gate=None, alpha=1.0):
    """Gradients of sum(dy * y) + sum(dh * h): dict name -> (value, size).  dgate has the gate's broadcast shape."""
    x = np.asarray(x, np.float64)
    M, H = x.shape
    g = np.ones((1, 1)) if gate is None else np.asarray(gate, np.float64)
    y, _, size_y, _ = forward(x, r, w_pre, eps, w_post, gate, alpha)
    rx = _rms(x, eps)
    xh = x * rx
    b = x if w_post is None else xh * w_post
    d = np.zeros((M, H)) if dy is None else np.asarray(dy, np.float64).copy()
    size_d = np.abs(d)
    out = {}
    if dh is not None:
        dh = np.asarray(dh, np.float64)
        ry = _rms(y, eps)
        yh = y * ry
        spread = 1.0 + np.sqrt(np.mean(size_y ** 2, axis=1, keepdims=True)) * ry
        size_yh = size_y * ry * spread
        t = dh * w_pre
        d += ry * (t - yh * np.mean(t * yh, axis=1, keepdims=True))
        size_d += ry * spread * (np.abs(t) + size_yh * np.mean(np.abs(t) * size_yh, axis=1, keepdims=True))
        out["dw_pre"] = ((dh * yh).sum(0), (np.abs(dh) * size_yh).sum(0))
    if r is not None:
        out["dr"] = (alpha * d, np.abs(alpha) * size_d)
    if gate is not None:
        e, se = d * b, size_d * np.abs(b)
        if g.shape == (M, H):
            out["dgate"] = (e, se)
        elif g.ndim == 2 and g.shape[1] == 1:
            out["dgate"] = (e.sum(1), se.sum(1))
        else:
            out["dgate"] = (e.sum(0), se.sum(0))
    db, size_db = g * d, np.abs(g) * size_d
    if w_post is None:
        out["dx"] = (db, size_db)
    else:
        t, st = db * w_post, size_db * np.abs(w_post)
        out["dx"] = (rx * (t - xh * np.mean(t * xh, axis=1, keepdims=True)),
                     rx * (st + np.abs(xh) * np.mean(st * np.abs(xh), axis=1, keepdims=True)))
        out["dw_post"] = ((db * xh).sum(0), (size_db * np.abs(xh)).sum(0))
    return out
