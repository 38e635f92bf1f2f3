"""The block norm's oracle against central differences and against cases known in closed form (CPU), and the entry
points' refusals, which need no device."""
import ctypes

import numpy as np
import pytest

from oracle import norm_oracle as nor
from paper_2502_16880_b200 import build as cbuild
from paper_2502_16880_b200 import lmhead


def _case(seed, M=3, H=16, post=True, gate="channel", residual=True):
    rng = np.random.default_rng(seed)
    g = {"none": None, "channel": rng.normal(size=H), "row": rng.normal(size=(M, 1)), "full": rng.normal(size=(M, H))}[gate]
    return dict(x=rng.normal(size=(M, H)), r=rng.normal(size=(M, H)) if residual else None, w_pre=1 + rng.normal(size=H),
                w_post=1 + rng.normal(size=H) if post else None, gate=g), rng.normal(size=(M, H)), rng.normal(size=(M, H))


def test_forward_closed_forms():
    x = np.full((2, 8), 3.0)
    y, h, _, _ = nor.forward(x, None, np.ones(8), 0.0)
    assert np.allclose(y, 3.0) and np.allclose(h, 1.0)                      # a constant row has root mean square 3
    y, h, _, _ = nor.forward(x, -3.0 * np.ones((2, 8)), np.ones(8), 1e-5)
    assert np.all(y == 0) and np.all(h == 0)
    y, _, _, _ = nor.forward(x, x, np.ones(8), 0.0, w_post=2 * np.ones(8), gate=np.full((2, 1), 0.5), alpha=0.25)
    assert np.allclose(y, 0.75 + 1.0)


@pytest.mark.parametrize("gate", ["none", "channel", "row", "full"])
@pytest.mark.parametrize("post", [False, True])
def test_gradient_against_central_differences(post, gate):
    inp, dy, dh = _case(5 + post, post=post, gate=gate)
    eps, alpha, step = 1e-3, 0.6, 1e-5

    def loss(**kw):
        y, h, _, _ = nor.forward(kw["x"], kw["r"], kw["w_pre"], eps, kw["w_post"], kw["gate"], alpha)
        return float((dy * y).sum() + (dh * h).sum())

    grads = nor.backward(inp["x"], inp["r"], inp["w_pre"], eps, dy, dh, inp["w_post"], inp["gate"], alpha)
    for leaf, name in [("x", "dx"), ("r", "dr"), ("w_pre", "dw_pre"), ("w_post", "dw_post"), ("gate", "dgate")]:
        if inp[leaf] is None:
            assert name not in grads
            continue
        want = np.empty(inp[leaf].size)
        for i in range(want.size):
            lo, hi = inp[leaf].copy(), inp[leaf].copy()
            lo.reshape(-1)[i] -= step
            hi.reshape(-1)[i] += step
            want[i] = (loss(**{**inp, leaf: hi}) - loss(**{**inp, leaf: lo})) / (2 * step)
        # truncation O(step^2), rounding of the loss 1e-15 / step
        assert np.allclose(grads[name][0].reshape(-1), want, rtol=1e-6, atol=1e-7), name


def test_one_gradient_absent_is_a_zero_gradient():
    inp, dy, dh = _case(9, gate="full")
    zero = np.zeros_like(dy)
    a = nor.backward(inp["x"], inp["r"], inp["w_pre"], 1e-5, dy, zero, inp["w_post"], inp["gate"])
    b = nor.backward(inp["x"], inp["r"], inp["w_pre"], 1e-5, dy, None, inp["w_post"], inp["gate"])
    for k in b:
        assert np.array_equal(a[k][0], b[k][0])


# ---- refusals: every argument error is found before anything reaches the device ------------------------------
def _args(**kw):
    p = 0x10000                                            # aligned, never dereferenced: each call below is refused
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_norm_args), type=lmhead.CORAL_TYPE_BF16, M=2, H=16, gate_mode=0,
                alpha=1.0, eps=1e-5, x_dev=p, r_dev=p, w_pre_dev=p, out_y_dev=p, out_h_dev=p, dy_dev=p, dh_dev=p, out_dx_dev=p,
                out_dr_dev=p, out_dw_pre_dev=p)
    base.update(kw)
    return lmhead.coral_lmhead_norm_args(**base)


BAD = [dict(struct_size=8), dict(type=3), dict(type=-1), dict(M=0), dict(M=-1), dict(H=12), dict(H=0), dict(H=16392),
       dict(type=0, H=8200), dict(gate_mode=4), dict(gate_mode=-1), dict(gate_mode=1), dict(gate_dev=0x10000), dict(eps=-1.0),
       dict(eps=float("nan")), dict(x_dev=None), dict(x_dev=0x10008), dict(r_dev=0x10002), dict(w_post_dev=0x10004),
       dict(gate_mode=1, gate_dev=0x10002), dict(gate_mode=2, gate_dev=0x10001)]


@pytest.mark.parametrize("kw", BAD + [dict(out_y_dev=None, out_h_dev=None), dict(w_pre_dev=None), dict(out_y_dev=0x10008),
                                      dict(out_h_dev=0x10002)])
def test_forward_refusals(kw):
    cbuild.build_library()
    a = _args(**kw)
    assert lmhead.load_library().coral_lmhead_block_norm(ctypes.byref(a), None) == lmhead.CORAL_ERR_INVALID


@pytest.mark.parametrize("kw", BAD + [dict(out_dx_dev=None), dict(dy_dev=None, dh_dev=None), dict(w_pre_dev=None, out_dw_pre_dev=None),
                                      dict(r_dev=None), dict(out_dw_post_dev=0x10000), dict(out_dgate_dev=0x10000),
                                      dict(dy_dev=None, dh_dev=None, w_pre_dev=None, out_dw_pre_dev=None), dict(out_dx_dev=0x10008),
                                      dict(out_dw_pre_dev=0x10002), dict(dh_dev=0x10008)])
def test_backward_refusals(kw):
    cbuild.build_library()
    a = _args(**kw)
    f = lmhead.load_library().coral_lmhead_block_norm_backward
    assert f(ctypes.byref(a), ctypes.c_void_p(0x10000), None) == lmhead.CORAL_ERR_INVALID


def test_backward_refuses_a_bad_workspace_and_sizes():
    cbuild.build_library()
    f = lmhead.load_library().coral_lmhead_block_norm_backward
    for w in (None, 0x10010):
        assert f(ctypes.byref(_args()), ctypes.c_void_p(w), None) == lmhead.CORAL_ERR_INVALID
    assert f(None, ctypes.c_void_p(0x10000), None) == lmhead.CORAL_ERR_INVALID
    for M, H in [(0, 16), (1, 12), (1, 0), (1, 16392)]:
        with pytest.raises(lmhead.CoralError) as e:
            lmhead.coral_lmhead_block_norm_backward_bytes(M, H)
        assert e.value.code == lmhead.CORAL_ERR_INVALID
    assert lmhead.coral_lmhead_block_norm_backward_bytes(1, 16) == 3 * 16 * 4
    a, b = (lmhead.coral_lmhead_block_norm_backward_bytes(m, 4096) for m in (10000, 1000000))
    assert a == b                                          # bounded by the device, not by the rows
