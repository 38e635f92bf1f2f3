"""GPU parity of the block norm and its gradient against the float64 oracle.

Tolerances.  u = 2^-24.  A thread adds at most 8 * 4 squares, a warp 5 partial sums, a block 16: a mean square is off by at
most 53 u relative, its reciprocal square root by half of that plus 2 u, the products behind it by 4 u more.  Each result is
therefore within C u of `size`, the formula over absolute values that the oracle returns (C = 64 forward, where one norm feeds
another; 256 backward, where two norms and three sums follow one another), plus one rounding to the output's type.  A sum
over M rows adds at most M u relative to its own size.
"""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as nor
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}      # half a step of the subnormals
MODE = {"none": 0, "channel": 1, "row": 2, "full": 3}


def _make(seed, M, H, t, post, gate, residual=True, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: (torch.randn(*s, generator=g) * scale).to(t)
    d = dict(x=rnd(M, H), r=rnd(M, H) if residual else None, w_pre=(1 + 0.3 * torch.randn(H, generator=g)).to(t),
             w_post=(1 + 0.3 * torch.randn(H, generator=g)).to(t) if post else None,
             gate={"none": None, "channel": rnd(H), "row": rnd(M), "full": rnd(M, H)}[gate], dy=rnd(M, H), dh=rnd(M, H))
    return d


def _np(t):
    return None if t is None else t.double().numpy()


def _gate_np(d, mode):
    return _np(d["gate"])[:, None] if mode == "row" else _np(d["gate"])


def _cuda(d):
    return {k: None if v is None else v.cuda() for k, v in d.items()}


def _forward(c, mode, alpha, eps, want_y=True, want_h=True, stream=None):
    y = torch.empty_like(c["x"]) if want_y else None
    h = torch.empty_like(c["x"]) if want_h else None
    lmhead.coral_lmhead_block_norm(c["x"], c["r"], c["w_pre"], eps, y, h, w_post=c["w_post"], gate=c["gate"],
                                   gate_mode=MODE[mode], alpha=alpha, stream=stream)
    return y, h


def _backward(c, mode, alpha, eps, dy=True, dh=True):
    M, H = c["x"].shape
    f = lambda *s: torch.full(s, 7.0, dtype=torch.float32, device="cuda")
    out = dict(dx=torch.empty_like(c["x"]), dr=None if c["r"] is None else torch.empty_like(c["x"]),
               dw_pre=f(H) if dh else None, dw_post=None if c["w_post"] is None else f(H),
               dgate={"none": None, "channel": f(H), "row": f(M), "full": torch.empty_like(c["x"])}[mode])
    ws = torch.full((lmhead.coral_lmhead_block_norm_backward_bytes(M, H),), 255, dtype=torch.uint8, device="cuda")
    lmhead.coral_lmhead_block_norm_backward(
        c["x"], c["r"], c["w_pre"], eps, c["dy"] if dy else None, c["dh"] if dh else None, ws, out["dx"], out["dr"], out["dw_pre"],
        w_post=c["w_post"], gate=c["gate"], gate_mode=MODE[mode], alpha=alpha, out_dw_post=out["dw_post"], out_dgate=out["dgate"])
    return out


def _close(got, want, size, C, what):
    t = got.dtype
    tol = C * U * size + torch.finfo(t).eps / 2 * (np.abs(want) + C * U * size) + TINY[t]
    off = np.abs(got.double().cpu().numpy() - want)
    assert np.all(off <= tol), (what, float(np.max(off / np.maximum(tol, 1e-300))))


SHAPES = [(1, 8), (1, 4096), (3, 264), (7, 3584), (333, 256), (1030, 72), (5, 4104), (9, 8192)]
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M,H", SHAPES)
def test_forward_and_gradient(M, H, t):
    for i, (post, mode) in enumerate([(False, "none"), (True, "channel"), (False, "row"), (True, "full"), (True, "row"), (False, "channel")]):
        if M * H > 40000 and i not in (1, 2, 3):
            continue
        d = _make(M * 31 + H + i, M, H, t, post, mode)
        c, alpha, eps = _cuda(d), 0.75, 1e-5
        y, h = _forward(c, mode, alpha, eps)
        wy, wh, sy, sh = nor.forward(_np(d["x"]), _np(d["r"]), _np(d["w_pre"]), eps, _np(d["w_post"]), _gate_np(d, mode), alpha)
        _close(y, wy, sy, 64, ("y", post, mode))
        _close(h, wh, sh, 64, ("h", post, mode))
        got = _backward(c, mode, alpha, eps)
        want = nor.backward(_np(d["x"]), _np(d["r"]), _np(d["w_pre"]), eps, _np(d["dy"]), _np(d["dh"]), _np(d["w_post"]),
                            _gate_np(d, mode), alpha)
        for k, (v, s) in want.items():
            summed = k in ("dw_pre", "dw_post") or (k == "dgate" and mode in ("channel", "row"))
            _close(got[k], v, s, 256 + (M if summed else 0), (k, post, mode))


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
def test_widest_rows(t):
    d = _make(3, 3, 16384, t, True, "full")
    c = _cuda(d)
    y, h = _forward(c, "full", 1.0, 1e-6)
    wy, wh, sy, sh = nor.forward(_np(d["x"]), _np(d["r"]), _np(d["w_pre"]), 1e-6, _np(d["w_post"]), _np(d["gate"]))
    _close(y, wy, sy, 64, "y")
    _close(h, wh, sh, 64, "h")
    got = _backward(c, "full", 1.0, 1e-6)
    want = nor.backward(_np(d["x"]), _np(d["r"]), _np(d["w_pre"]), 1e-6, _np(d["dy"]), _np(d["dh"]), _np(d["w_post"]), _np(d["gate"]))
    for k, (v, s) in want.items():
        _close(got[k], v, s, 256 + 3, k)


def test_absent_parts():
    """No residual, no second norm, only one output, only one incoming gradient."""
    t, M, H, eps = torch.bfloat16, 5, 512, 1e-5
    d = _make(11, M, H, t, True, "channel", residual=False)
    c = _cuda(d)
    y, h = _forward(c, "channel", 0.3, eps)
    wy, wh, sy, sh = nor.forward(_np(d["x"]), None, _np(d["w_pre"]), eps, _np(d["w_post"]), _np(d["gate"]), 0.3)
    _close(y, wy, sy, 64, "y")
    _close(h, wh, sh, 64, "h")
    only_h = _forward(c, "channel", 0.3, eps, want_y=False)[1]
    assert torch.equal(only_h, h)
    d = _make(12, M, H, t, False, "none")
    c = _cuda(d)
    for dy, dh in [(True, False), (False, True)]:
        got = _backward(c, "none", 0.7, eps, dy=dy, dh=dh)
        want = nor.backward(_np(d["x"]), _np(d["r"]), _np(d["w_pre"]), eps, _np(d["dy"]) if dy else None, _np(d["dh"]) if dh else None,
                            None, None, 0.7)
        for k, (v, s) in want.items():
            _close(got[k], v, s, 256 + M, (k, dy, dh))
    c["w_pre"] = None
    y2, _ = _forward(c, "none", 0.7, eps, want_h=False)
    wy, _, sy, _ = nor.forward(_np(d["x"]), _np(d["r"]), None, eps, None, None, 0.7)
    _close(y2, wy, sy, 64, "y without the second norm")


def test_special_rows():
    """A row of zeros stays zero with eps > 0; huge and tiny rows keep their scale out of h; NaN stays in its row."""
    t, H = torch.float32, 1024
    d = _make(4, 6, H, t, False, "none", residual=False)
    d["x"][0] = 0
    d["x"][1] *= 1e15
    d["x"][2] *= 1e-15
    d["x"][3, 5] = float("nan")
    c = _cuda(d)
    y, h = _forward(c, "none", 1.0, 1e-38)
    y, h = y.cpu(), h.cpu()
    assert torch.all(h[0] == 0) and torch.all(torch.isnan(h[3])) and int(torch.isnan(y[3]).sum()) == 1
    for m in (1, 2, 4, 5):
        _, wh, _, sh = nor.forward(_np(d["x"][m:m + 1]), None, _np(d["w_pre"]), 1e-38)
        _close(h[m:m + 1], wh, sh, 64, m)
    zero = torch.zeros(1, H, device="cuda")
    out = torch.empty_like(zero)
    lmhead.coral_lmhead_block_norm(zero, None, c["w_pre"], 0.0, None, out)
    assert torch.all(torch.isnan(out))                                      # 0 / 0, as the formula has it


def test_in_place_other_stream_repeat_and_graph():
    t, M, H, eps = torch.bfloat16, 700, 1024, 1e-5
    c = _cuda(_make(21, M, H, t, True, "full"))
    y, h = _forward(c, "full", 0.9, eps)
    first = _backward(c, "full", 0.9, eps)
    again = _backward(c, "full", 0.9, eps)
    for k in first:
        if first[k] is not None:
            assert torch.equal(first[k], again[k]), k                       # no order of additions is left to chance
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, h2 = _forward(c, "full", 0.9, eps, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2)
    x, r = c["x"].clone(), c["r"].clone()
    lmhead.coral_lmhead_block_norm(x, r, c["w_pre"], eps, r, x, w_post=c["w_post"], gate=c["gate"], gate_mode=3, alpha=0.9)
    assert torch.equal(r, y) and torch.equal(x, h)
    # gradient over its own inputs
    dy, dh = c["dy"].clone(), c["dh"].clone()
    ws = torch.empty(lmhead.coral_lmhead_block_norm_backward_bytes(M, H), dtype=torch.uint8, device="cuda")
    kw = dict(w_post=c["w_post"], gate=c["gate"], gate_mode=3, alpha=0.9)
    lmhead.coral_lmhead_block_norm_backward(c["x"], c["r"], c["w_pre"], eps, dy, dh, ws, dh, dy, **kw)
    assert torch.equal(dh, first["dx"]) and torch.equal(dy, first["dr"])
    # forward and backward captured, replayed on new inputs in the same buffers
    y3, h3, dx, dr = (torch.empty_like(y) for _ in range(4))
    dwp = torch.empty(H, device="cuda")

    def both():
        lmhead.coral_lmhead_block_norm(c["x"], c["r"], c["w_pre"], eps, y3, h3, **kw)
        lmhead.coral_lmhead_block_norm_backward(c["x"], c["r"], c["w_pre"], eps, c["dy"], c["dh"], ws, dx, dr, dwp, **kw)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    c["x"].mul_(1.5)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    got = [v.clone() for v in (y3, h3, dx, dr, dwp)]
    both()
    torch.cuda.synchronize()
    for a, b in zip(got, (y3, h3, dx, dr, dwp)):
        assert torch.equal(a, b)


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    o = torch.empty_like(x)
    call = lmhead.coral_lmhead_block_norm
    for bad in [dict(r=x.float()), dict(r=x[:2]), dict(r=torch.zeros(4, 128, device="cuda", dtype=torch.bfloat16)[:, ::2]), dict(r=x.cpu()),
                dict(gate=w), dict(gate=w, gate_mode=2), dict(gate_mode=1), dict(w_post=w[:32])]:
        kw = dict(r=x)
        kw.update(bad)
        with pytest.raises((ValueError, lmhead.CoralError)):
            call(x, kw.pop("r"), w, 1e-5, o, o.clone(), **kw)
    with pytest.raises(ValueError):
        call(x.to(torch.int32), None, w, 1e-5, o, o)
    with pytest.raises(ValueError):                                          # a workspace that is too small
        lmhead.coral_lmhead_block_norm_backward(x, x, w, 1e-5, x, x, torch.empty(16, dtype=torch.uint8, device="cuda"), o)
