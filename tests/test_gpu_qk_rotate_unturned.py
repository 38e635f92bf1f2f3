"""Norm and rotation of queries and keys: columns that are not turned go by themselves, whatever stands in the others."""
import pytest
import torch

from tests.test_gpu_qk_rotate import TYPES, _backward, _forward, _make

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
SHAPES = [(64, 32), (128, 64), (96, 8), (40, 0), (72, 24), (256, 128), (128, 112)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("D,rot", SHAPES)
def test_without_a_norm(D, rot, style, t):
    """y = x and dx = dout there, bit for bit, beside an infinity or a NaN too (which itself comes through)."""
    d = _make(D, 9, 5, 2, D, rot, t, (False, False))
    x = {n: d[n].clone() for n in ("q", "k", "dq", "dk")}
    for bad in (INF, -INF, NAN):
        for c in {rot, rot + 3, (rot + D) // 2, D - 1}:
            for n in x:
                d[n] = x[n].clone()
                d[n][3, 1, c] = bad
            out, back = _forward(d, style), _backward(d, style)
            for got, want in ((out[0], d["q"]), (out[1], d["k"]), (back["dq"], d["dq"]), (back["dk"], d["dk"])):
                same = got[..., rot:].eq(want[..., rot:]) | (got[..., rot:].isnan() & want[..., rot:].isnan())
                assert same.all() and got[..., :rot].isfinite().all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("D,rot", [s for s in SHAPES if s[1]])
def test_with_a_norm(D, rot, style, t):
    """An infinity makes its row's root infinite: NaN in its own column, zero in the others; one in the weights stays in its column."""
    d = _make(D + 1, 9, 5, 2, D, rot, t)
    c = (rot + D) // 2
    rest = [i for i in range(D) if i != c]
    d["q"], d["k"] = d["q"].clone(), d["k"].clone()
    d["q"][3, 1, c] = d["k"][3, 1, c] = INF
    for y in _forward(d, style):
        assert y[3, 1, c].isnan() and not y[3, 1, rest].any()
    d["q"][3, 1, c] = d["k"][3, 1, c] = 1.0
    want = _forward(d, style)
    d["w_q"][c] = d["w_k"][c] = INF
    for y, w in zip(_forward(d, style), want):
        assert y[..., c].isinf().all() and torch.equal(y[..., rest], w[..., rest])
