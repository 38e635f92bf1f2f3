"""GPU parity of the norm and rotation of queries and keys, and of their gradient, against the float64 oracle.

Tolerances.  u = 2^-24.  A mean square of up to 256 columns: a thread adds 16 squares, five shuffle steps follow: 23 u, half of that in its
root, 3 u for root, quotient and eps; the products behind it 2 u.  An angle in turns is rounded to fp32 once (pi u at most), its sine and
cosine are off by 2 u more: 6 u of |a| + |b|; two products and a sum 3 u.  Forward 12 + 3 + 2 + 6 + 3 < C = 32 times u times the size.
Backward: the turn (9 u), r twice (30 u), a mean of products (9 + 15 + 25 u), products 6 u: C = 128.  A sum over n rows: C + n.
One rounding to the output's type comes on top."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2502_16880_b200 import lmhead

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
EPS = 1e-6


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _freqs(rot, base=10000.0):
    return (base ** -(torch.arange(0, rot, 2).double() / max(rot, 1))).float()


def _make(seed, T, n_q, n_k, D, rot, t, norm=(True, True), far=0, extra=0):
    g = torch.Generator().manual_seed(seed)
    fused = (torch.randn(T, n_q + 2 * n_k + extra, D, generator=g) * 1.5).to(t).cuda()
    d = dict(q=fused[:, :n_q] if n_q else None, k=fused[:, n_q:n_q + n_k] if n_k else None, positions=(torch.arange(T) + far).int().cuda(),
             freqs=_freqs(rot).cuda() if rot else None)
    for n, on in zip(("w_q", "w_k"), norm):
        d[n] = (1 + 0.3 * torch.randn(D, generator=g)).to(t).cuda() if on and (n_q if n == "w_q" else n_k) else None
    for n, h in (("q", n_q), ("k", n_k)):
        d["d" + n] = torch.randn(T, h, D, generator=g).to(t).cuda() if h else None
    return d


def _close(got, want, size, C, what):
    t = got.dtype
    tol = C * U * size + torch.finfo(t).eps / 2 * (np.abs(want) + C * U * size) + TINY[t]
    off = np.abs(_np(got) - want)
    assert np.all(off <= tol), (what, float(np.max(off / np.maximum(tol, 1e-300))))


def _forward(d, style, out_q=None, out_k=None, **kw):
    new = lambda x: None if x is None else torch.empty(x.shape, dtype=x.dtype, device="cuda")
    out_q, out_k = new(d["q"]) if out_q is None else out_q, new(d["k"]) if out_k is None else out_k
    lmhead.coral_lmhead_qk_rotate(d["q"], d["k"], d["positions"], d["freqs"], out_q, out_k, w_q=d["w_q"], w_k=d["w_k"], eps=EPS, style=style, **kw)
    return out_q, out_k


def _backward(d, style, dq=None, dk=None, **kw):
    new = lambda x: None if x is None else torch.empty_like(x)
    f = lambda w, D: None if w is None else torch.full((D,), 7.0, device="cuda")
    first = d["dq"] if d["dq"] is not None else d["dk"]
    T, D = first.shape[0], first.shape[2]
    n = [0 if d[x] is None else d[x].shape[1] for x in ("dq", "dk")]
    ws = torch.full((lmhead.coral_lmhead_qk_rotate_backward_bytes(T, *n, D),), 255, dtype=torch.uint8, device="cuda")
    out = dict(dq=new(d["dq"]) if dq is None else dq, dk=new(d["dk"]) if dk is None else dk, dw_q=f(d["w_q"], D), dw_k=f(d["w_k"], D))
    lmhead.coral_lmhead_qk_rotate_backward(d["q"], d["k"], d["positions"], d["freqs"], d["dq"], d["dk"], out["dq"], out["dk"], w_q=d["w_q"], w_k=d["w_k"],
                                           eps=EPS, style=style, dw_q=out["dw_q"], dw_k=out["dw_k"], workspace=ws, **kw)
    return out


def _check(d, style):
    f, pos = [] if d["freqs"] is None else _np(d["freqs"]), d["positions"].cpu().numpy()
    got = _forward(d, style)
    for n, y in zip("qk", got):
        if d[n] is not None:
            _close(y, *ao.qk(_np(d[n]), _np(d["w_" + n]), pos, f, style == 1, EPS), 32, n)
    back = _backward(d, style)
    for n in "qk":
        if d[n] is None:
            continue
        (dx, size), more = ao.qk_backward(_np(d[n]), _np(d["w_" + n]), pos, f, style == 1, EPS, _np(d["d" + n]))
        _close(back["d" + n], dx, size, 128, "d" + n)
        if more is not None:
            _close(back["dw_" + n], *more, 128 + d[n].shape[0] * d[n].shape[1], "dw_" + n)


SHAPES = [(1, 1, 1, 8, 8), (1, 28, 4, 128, 128), (3, 4, 2, 64, 32), (17, 3, 1, 96, 88), (5, 7, 7, 256, 256), (130, 8, 2, 128, 64), (9, 5, 3, 72, 24),
          (33, 2, 2, 40, 0), (700, 12, 3, 128, 128), (2, 33, 1, 248, 8), (611, 1, 1, 16, 16)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("T,n_q,n_k,D,rot", SHAPES)
def test_forward_and_gradient(T, n_q, n_k, D, rot, style, t):
    _check(_make(T * 7 + D, T, n_q, n_k, D, rot, t, far=3 * T), style)


@pytest.mark.parametrize("norm", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("n_q,n_k", [(4, 2), (4, 0), (0, 2)])
def test_parts_left_out(n_q, n_k, norm):
    for style in (0, 1):
        _check(_make(5, 19, n_q, n_k, 64, 48, torch.float32, norm), style)


def test_no_norm_needs_no_input_for_its_gradient():
    d = _make(6, 21, 4, 2, 64, 64, torch.bfloat16, (False, False))
    want = _backward(d, 0)
    d["q"] = d["k"] = None
    got = _backward(d, 0)
    assert torch.equal(got["dq"], want["dq"]) and torch.equal(got["dk"], want["dk"])


@pytest.mark.parametrize("style", [0, 1])
def test_far_and_negative_positions(style):
    d = _make(8, 6, 2, 1, 64, 64, torch.float32)
    d["positions"] = torch.tensor([0, -1, 1000003, -1000003, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    _check(d, style)


def test_in_place_and_strided_outputs():
    for style in (0, 1):
        d = _make(9, 50, 6, 2, 128, 96, torch.bfloat16)
        want, grads = _forward(d, style), _backward(d, style)
        room = torch.full((50, 11, 128), 3.0, dtype=torch.bfloat16, device="cuda")
        _forward(d, style, room[:, 1:7], room[:, 8:10])
        assert torch.equal(room[:, 1:7], want[0]) and torch.equal(room[:, 8:10], want[1])
        assert (room[:, 0] == 3).all() and (room[:, 7] == 3).all() and (room[:, 10] == 3).all()
        got = _backward(d, style, room[:, 1:7], room[:, 8:10])
        assert torch.equal(room[:, 1:7], grads["dq"]) and torch.equal(room[:, 8:10], grads["dk"]) and torch.equal(got["dw_q"], grads["dw_q"])
        same = dict(d, q=d["q"].clone(), k=d["k"].clone())
        got = _backward(same, style, same["q"], same["k"])                       # gradients over the inputs
        assert torch.equal(got["dq"], grads["dq"]) and torch.equal(got["dk"], grads["dk"])
        same = dict(d, dq=d["dq"].clone(), dk=d["dk"].clone())
        _backward(same, style, same["dq"], same["dk"])                           # ... and over the gradients that came in
        assert torch.equal(same["dq"], grads["dq"]) and torch.equal(same["dk"], grads["dk"])
        values = d["q"].as_strided((50, 2, 128), d["q"].stride(), d["q"].storage_offset() + 8 * 128).clone()
        _forward(d, style, d["q"], d["k"])                                       # over the fused projection itself
        assert torch.equal(d["q"], want[0]) and torch.equal(d["k"], want[1])
        assert torch.equal(values, d["q"].as_strided((50, 2, 128), d["q"].stride(), d["q"].storage_offset() + 8 * 128))


def test_a_bad_row_stays_in_its_row():
    d = _make(10, 40, 4, 2, 64, 64, torch.bfloat16)
    want = _forward(d, 0)
    back = _backward(d, 0)
    d["q"][7, 2, 5], d["k"][8, 1, 3] = float("nan"), float("inf")
    got, grads = _forward(d, 0), _backward(d, 0)
    keep_q, keep_k = torch.ones(40, 4, dtype=torch.bool), torch.ones(40, 2, dtype=torch.bool)
    keep_q[7, 2] = keep_k[8, 1] = False
    for g, w in ((got[0], want[0]), (grads["dq"], back["dq"])):
        assert torch.equal(g[keep_q], w[keep_q]) and not g[7, 2].isfinite().any()
    for g, w in ((got[1], want[1]), (grads["dk"], back["dk"])):
        assert torch.equal(g[keep_k], w[keep_k]) and g[8, 1].isnan().any()


def test_gradient_against_differences():
    """Of the kernel's own forward pass, in fp32: a loss of h-wide differences is off by the forward's 32 u of its size over h, and by h^2
    of the third derivative."""
    d = _make(11, 4, 2, 1, 16, 16, torch.float32)
    back, h = _backward(d, 0), 2.0 ** -6
    probe = torch.Generator().manual_seed(1)
    for n, i in (("q", 0), ("k", 1)):
        e = torch.randn(d[n].shape, generator=probe).cuda()
        e = e / e.norm()
        at = []
        for s in (h, -h):
            moved = dict(d)
            moved[n] = (d[n] + s * e).contiguous()
            at.append((_forward(moved, 0)[i].double() * d["d" + n].double()).sum().item())
        size = (_forward(d, 0)[i].double().abs() * d["d" + n].double().abs()).sum().item()
        want = (back["d" + n].double() * e.double()).sum().item()
        assert abs((at[0] - at[1]) / (2 * h) - want) <= 2 * 64 * U * size / h + 10 * h * h * d["d" + n].norm().item()


@pytest.mark.parametrize("T", [1, 400, 5000])
def test_repeat_streams_and_graph(T):
    d = _make(12, T, 8, 2, 128, 128, torch.bfloat16)
    want, grads = _forward(d, 0), _backward(d, 0)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got, back = _forward(d, 0, stream=st), _backward(d, 0, stream=st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(back[n], grads[n]) for n in grads)
    out, res = [torch.empty_like(x) for x in want], {n: torch.empty_like(x) for n, x in grads.items()}
    ws = torch.empty(lmhead.coral_lmhead_qk_rotate_backward_bytes(T, 8, 2, 128), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _forward(d, 0, *out)
        lmhead.coral_lmhead_qk_rotate_backward(d["q"], d["k"], d["positions"], d["freqs"], d["dq"], d["dk"], res["dq"], res["dk"], w_q=d["w_q"], w_k=d["w_k"],
                                               eps=EPS, dw_q=res["dw_q"], dw_k=res["dw_k"], workspace=ws)
    for _ in range(3):
        for x in (*out, *res.values()):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(res[n], grads[n]) for n in grads)


def test_binding_refuses_wrong_tensors():
    d = _make(13, 6, 4, 2, 64, 64, torch.bfloat16)
    for bad in (dict(q=d["q"].float()), dict(k=d["k"][:5]), dict(positions=d["positions"].long()), dict(positions=d["positions"][:5]),
                dict(freqs=d["freqs"].double()), dict(w_q=d["w_q"].float()), dict(w_k=d["w_k"][:32]), dict(q=d["q"].cpu()), dict(q=d["q"].transpose(1, 2)),
                dict(q=d["q"][:1].expand(6, 4, 64)), dict(freqs=torch.ones(33, device="cuda")), dict(freqs=torch.ones(2, device="cuda"))):
        with pytest.raises((ValueError, lmhead.CoralError)):
            _forward(dict(d, **bad), 0, torch.empty(6, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 2, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        lmhead.coral_lmhead_qk_rotate_backward(d["q"], d["k"], d["positions"], d["freqs"], d["dq"], d["dk"], torch.empty_like(d["dq"]), torch.empty_like(d["dk"]),
                                               w_q=d["w_q"], w_k=d["w_k"], dw_q=torch.empty(64, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_rows_beyond_32_bit_offsets():
    """Tokens 2^20 elements apart, the last of them 2^31 elements from the first: the same bits as side by side, both ways."""
    g = torch.Generator().manual_seed(5)
    T, n_q, n_k, D, t = 2100, 3, 2, 64, torch.bfloat16
    room = torch.empty(T, 2 ** 20, dtype=t, device="cuda")
    near = {n: torch.randn(T, h, D, generator=g).to(t).cuda() for n, h in (("q", n_q), ("k", n_k), ("dq", n_q), ("dk", n_k))}
    far = {}
    for i, (n, x) in enumerate(near.items()):
        far[n] = room[:, i * 256:i * 256 + x.shape[1] * D].view(x.shape)
        far[n].copy_(x)
    w = torch.randn(2, D, generator=g).to(t).cuda()
    pos, freqs = torch.arange(T, dtype=torch.int32, device="cuda") * 50, (10000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
    ws = torch.empty(lmhead.coral_lmhead_qk_rotate_backward_bytes(T, n_q, n_k, D), dtype=torch.uint8, device="cuda")
    got = []
    for x in (near, far):
        dw = [torch.empty(D, device="cuda") for _ in range(2)]
        lmhead.coral_lmhead_qk_rotate_backward(x["q"], x["k"], pos, freqs, x["dq"], x["dk"], x["dq"], x["dk"], w[0], w[1], dw_q=dw[0], dw_k=dw[1], workspace=ws)
        lmhead.coral_lmhead_qk_rotate(x["q"], x["k"], pos, freqs, x["q"], x["k"], w[0], w[1])
        got.append(dw + list(x.values()))
    assert all(torch.equal(a, b) for a, b in zip(*got))
