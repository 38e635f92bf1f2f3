"""Float64 oracles of the drafter's attention: norm and rotation of queries and keys, softmax attention over what a row sees, and
what a group of columns held in 4 bits stands for.  Written from the formulas in include/coral_lmhead.h; numpy, no blocking, no
fusion.  Next to a result stands its `size`: the same formula over absolute values, which rounding errors are relative to."""
import numpy as np


def _turn(a, b, angle):
    """A pair (a, b) turned: the product of a + ib with exp(i angle)."""
    z = (a + 1j * b) * np.exp(1j * angle)
    return z.real, z.imag


def rotate(x, positions, freqs, pairs, back=False):
    """x [T, heads, D]: its first 2 len(freqs) columns turned, pair by pair."""
    rot = 2 * len(freqs)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64)
    angle = (angle % (2 * np.pi))[:, None, :] * (-1 if back else 1)
    y = np.array(x, np.float64)
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first], y[..., second] = _turn(np.asarray(x[..., first], np.float64), np.asarray(x[..., second], np.float64), angle)
    return y


def _pair_size(x, rot, pairs):
    """|a| + |b| for both members of a turned pair, |x| elsewhere."""
    s = np.abs(np.asarray(x, np.float64))
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    both = s[..., first] + s[..., second]
    s[..., first] = s[..., second] = both
    return s


def qk(x, w, positions, freqs, pairs, eps):
    """(result, size) of norm (w [D], or None: none) and rotation."""
    n = np.asarray(x, np.float64)
    if w is not None:
        n = n / np.sqrt((n ** 2).mean(-1, keepdims=True) + eps) * w
    return rotate(n, positions, freqs, pairs), _pair_size(n, 2 * len(freqs), pairs)


def qk_backward(x, w, positions, freqs, pairs, eps, dy):
    """((dx, size), (dw, size) or None)."""
    d = rotate(dy, positions, freqs, pairs, back=True)
    d_size = _pair_size(dy, 2 * len(freqs), pairs)
    if w is None:
        return (d, d_size), None
    x = np.asarray(x, np.float64)
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    xh = r * x
    dx = r * (d * w - xh * (d * w * xh).mean(-1, keepdims=True))
    size = r * (d_size * np.abs(w) + np.abs(xh) * (d_size * np.abs(w * xh)).mean(-1, keepdims=True))
    return (dx, size), ((d * xh).sum((0, 1)), (d_size * np.abs(xh)).sum((0, 1)))


def attend(q, k, v, seen, scale):
    """q [Lq, n_q, D], k, v [Lk, n_k, D], seen [Lq, Lk]: out, lse, and per row and head the weights' sums of |v| [Lq, n_q, D], the
    largest size of a score (absolute products) [Lq, n_q], and how many keys a row sees [Lq].  Rows that see nothing: 0 and -inf."""
    Lq, n_q, D = q.shape
    n_k = k.shape[1]
    out, lse, vsize, ssize = np.zeros((Lq, n_q, D)), np.full((Lq, n_q), -np.inf), np.zeros((Lq, n_q, D)), np.zeros((Lq, n_q))
    for i in range(Lq):
        at = np.flatnonzero(seen[i])
        if not len(at):
            continue
        for h in range(n_q):
            kk, vv = np.asarray(k[at, h * n_k // n_q], np.float64), np.asarray(v[at, h * n_k // n_q], np.float64)
            s = kk @ np.asarray(q[i, h], np.float64) * scale
            m = s.max()
            p = np.exp(s - m)
            out[i, h], lse[i, h] = p @ vv / p.sum(), m + np.log(p.sum())
            vsize[i, h] = p @ np.abs(vv) / p.sum()
            ssize[i, h] = (np.abs(kk) @ np.abs(np.asarray(q[i, h], np.float64))).max() * abs(scale)
    return out, lse, vsize, ssize, seen.sum(1)


def causal(Lq, Lk):
    """Query i is key i + Lk - Lq and sees the keys up to itself."""
    return np.arange(Lk)[None, :] <= np.arange(Lq)[:, None] + Lk - Lq


def tree(masks, n, length):
    """The last n of `length` tokens are the queries; row i sees what is before them, and those whose bit in masks[i] is set."""
    seen = np.ones((n, length), bool)
    for i in range(n):
        for b in range(n):
            if length - n + b >= 0:
                seen[i, length - n + b] = int(masks[i]) >> b & 1
    return seen


def held(x, group, round_to_type):
    """x [..., D] in groups of columns: (low, step, codes, how far the nearest quotient lies from a border between two codes)."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, group)
    low = g.min(-1, keepdims=True)
    step = round_to_type((g.max(-1, keepdims=True) - low) / 15)
    with np.errstate(invalid="ignore", divide="ignore"):
        n = np.where(step > 0, (g - low) / np.where(step > 0, step, 1), 0)
    return low, step, np.clip(np.rint(n), 0, 15), np.abs(n - np.floor(n) - 0.5)


def stands_for(low, step, codes):
    return (low + step * codes).reshape(*codes.shape[:-2], -1)
