"""The oracles of the drafter's attention on cases known by hand and against differences (CPU), and the refusals of its entry
points, which need no device."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2502_16880_b200 import build as cbuild
from paper_2502_16880_b200 import lmhead

P = 0x10000                                                # aligned, never dereferenced: each call below is refused


@pytest.fixture(scope="module")
def lib():
    cbuild.build_library()
    return lmhead.load_library()


def test_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]])       # a quarter and a half turn
    f = [math.pi / 2, math.pi]
    assert np.allclose(ao.rotate(x, [1], f, False), [[[-3, -2, 1, -4, 5, 6]]])
    assert np.allclose(ao.rotate(x, [1], f, True), [[[-2, 1, -3, -4, 5, 6]]])
    assert np.allclose(ao.rotate(ao.rotate(x, [7], f, True), [7], f, True, back=True), x)
    y, size = ao.qk(np.array([[[3.0, 4.0]]]), np.array([1.0, 2.0]), [5], [], False, 0.0)
    assert np.allclose(y, np.array([[[3.0, 8.0]]]) / math.sqrt(12.5)) and np.allclose(size, np.abs(y))


def test_far_positions_turn_as_whole_numbers_say():
    p = 2 ** 31 - 1                                        # 2^31 - 1 quarter turns are 3 quarter turns past whole ones
    y = ao.rotate(np.array([[[1.0, 0.0]]]), [p], [math.pi / 2], True)
    assert np.allclose(y, [[[0.0, -1.0]]], atol=1e-6)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_gradient_against_differences(pairs, norm):
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    w = rng.standard_normal(8) if norm else None
    pos, f, eps, h = [0, 5, 9], [1.0, 0.3], 1e-3, 1e-6
    (dx, _), more = ao.qk_backward(x, w, pos, f, pairs, eps, dy)
    loss = lambda x, w: (ao.qk(x, w, pos, f, pairs, eps)[0] * dy).sum()
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[i]) < 1e-7
    if norm:
        for c in range(8):
            e = np.zeros(8)
            e[c] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - more[0][c]) < 1e-7


def test_attention_by_hand_and_against_torch():
    q, k, v = np.zeros((2, 1, 2)), np.zeros((3, 1, 2)), np.array([[[1.0, 0]], [[3.0, 0]], [[8.0, 6.0]]])
    out, lse, _, _, n = ao.attend(q, k, v, ao.causal(2, 3), 1.0)
    assert np.allclose(out[:, 0], [[2, 0], [4, 2]]) and np.allclose(lse[:, 0], np.log([2, 3])) and n.tolist() == [2, 3]
    out, lse, _, _, n = ao.attend(q, k[:1], v[:1], ao.causal(2, 1), 1.0)          # fewer keys than queries: the first sees none
    assert np.allclose(out[:, 0], [[0, 0], [1, 0]]) and lse[0, 0] == -np.inf and n.tolist() == [0, 1]
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    t = lambda x: torch.from_numpy(x).permute(1, 0, 2)
    want = torch.nn.functional.scaled_dot_product_attention(t(q), t(k).repeat_interleave(2, 0), t(v).repeat_interleave(2, 0),
                                                            attn_mask=torch.from_numpy(ao.causal(5, 9)), scale=0.3)
    out = ao.attend(q, k, v, ao.causal(5, 9), 0.3)[0]
    assert np.allclose(out, want.permute(1, 0, 2).numpy())
    assert ao.tree([0b001, 0b011, 0b101], 3, 4).tolist() == [[1, 1, 0, 0], [1, 1, 1, 0], [1, 1, 0, 1]]
    assert ao.tree([1, 3, 7], 3, 2).tolist() == [[0, 0], [1, 0], [1, 1]]            # a sequence shorter than its queries


def test_held_by_hand():
    low, step, codes, _ = ao.held(np.array([0.0, 1.0, 7.4, 15.0, 2.0, 2.0, 2.0, 2.0]), 4, lambda v: v)
    assert low.ravel().tolist() == [0, 2] and step.ravel().tolist() == [1, 0] and codes.tolist() == [[0, 1, 7, 15], [0, 0, 0, 0]]
    assert ao.stands_for(low, step, codes).tolist() == [0, 1, 7, 15, 2, 2, 2, 2]


# ---- refusals: every argument error is found before anything reaches the device ------------------------------
def _qk(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_qk_args), type=1, T=2, n_q=4, n_k=2, D=64, rot=32, style=0, eps=1e-6,
                ld_q=256, ld_k=128, ld_out_q=256, ld_out_k=128, ld_dout_q=256, ld_dout_k=128, ld_dq=256, ld_dk=128, q_dev=P, k_dev=P, w_q_dev=P,
                w_k_dev=P, positions_dev=P, freqs_dev=P, out_q_dev=P, out_k_dev=P, dout_q_dev=P, dout_k_dev=P, dq_dev=P, dk_dev=P)
    base.update(kw)
    return lmhead.coral_lmhead_qk_args(**base)


QK_BAD = [dict(struct_size=8), dict(type=3), dict(T=0), dict(T=-1), dict(n_q=-1), dict(n_q=0, n_k=0), dict(n_k=5000), dict(D=12), dict(D=0), dict(D=264),
          dict(rot=4), dict(rot=72), dict(rot=-8), dict(style=2), dict(style=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(positions_dev=None),
          dict(positions_dev=P + 2), dict(freqs_dev=None), dict(freqs_dev=P + 2), dict(w_q_dev=P + 8), dict(w_k_dev=P + 2), dict(q_dev=None),
          dict(k_dev=P + 8), dict(ld_q=255), dict(ld_q=260), dict(ld_k=120), dict(ld_q=-256)]


@pytest.mark.parametrize("kw", QK_BAD + [dict(out_q_dev=None), dict(out_k_dev=P + 4), dict(ld_out_q=248), dict(ld_out_k=132)])
def test_qk_refusals(lib, kw):
    assert lib.coral_lmhead_qk_rotate(ctypes.byref(_qk(**kw)), None) == lmhead.CORAL_ERR_INVALID


@pytest.mark.parametrize("kw", QK_BAD + [dict(dout_q_dev=None), dict(dk_dev=None), dict(dq_dev=P + 8), dict(ld_dq=248), dict(ld_dout_k=130),
                                         dict(dw_q_dev=P, w_q_dev=None), dict(dw_k_dev=P + 2), dict(dw_k_dev=P, n_k=0)])
def test_qk_backward_refusals(lib, kw):
    assert lib.coral_lmhead_qk_rotate_backward(ctypes.byref(_qk(**kw)), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID


def test_qk_backward_refuses_a_bad_workspace_and_sizes(lib):
    for ws in (None, P + 16):
        assert lib.coral_lmhead_qk_rotate_backward(ctypes.byref(_qk(dw_q_dev=P)), ctypes.c_void_p(ws), None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_qk_rotate(None, None) == lmhead.CORAL_ERR_INVALID
    for bad in [(0, 1, 1, 64), (1, 0, 0, 64), (1, -1, 2, 64), (1, 1, 1, 12), (1, 1, 1, 264)]:
        with pytest.raises(lmhead.CoralError):
            lmhead.coral_lmhead_qk_rotate_backward_bytes(*bad)
    assert lmhead.coral_lmhead_qk_rotate_backward_bytes(1, 4, 2, 64) == 2 * 64 * 4
    a, b = (lmhead.coral_lmhead_qk_rotate_backward_bytes(t, 4, 2, 64) for t in (10 ** 4, 10 ** 6))
    assert a == b


def _prompt(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_prompt_args), type=1, n_seq=1, T=4, Tk=4, n_q=4, n_k=2, D=64, scale=0.125, ld_q=256,
                ld_k=128, ld_v=128, ld_out=256, q_dev=P, k_dev=P, v_dev=P, q_offsets_dev=P, k_offsets_dev=P, out_dev=P, out_lse_dev=P)
    base.update(kw)
    return lmhead.coral_lmhead_prompt_args(**base)


@pytest.mark.parametrize("kw", [dict(struct_size=8), dict(type=0), dict(type=3), dict(n_seq=-1), dict(T=-1), dict(Tk=-1), dict(n_k=0), dict(n_q=3), dict(n_q=0),
                                dict(n_q=5000, n_k=5000), dict(D=4), dict(D=12), dict(D=136), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                                dict(scale=float("nan")), dict(q_dev=None), dict(k_dev=P + 8), dict(v_dev=None), dict(out_dev=P + 2), dict(q_offsets_dev=None),
                                dict(q_offsets_dev=P + 4), dict(k_offsets_dev=P + 4), dict(k_offsets_dev=None, Tk=5), dict(out_lse_dev=P + 2), dict(ld_q=248),
                                dict(ld_k=132), dict(ld_v=64), dict(ld_out=100)])
def test_prompt_refusals(lib, kw):
    assert lib.coral_lmhead_prompt_attention(ctypes.byref(_prompt(**kw)), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID


def test_prompt_refuses_a_bad_workspace_and_too_many_blocks(lib):
    for ws in (None, P + 16):
        assert lib.coral_lmhead_prompt_attention(ctypes.byref(_prompt()), ctypes.c_void_p(ws), None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_prompt_attention(None, ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID
    big = _prompt(T=2 ** 31 - 1, Tk=2 ** 31 - 1, n_q=4096, n_k=4096, ld_q=4096 * 64, ld_k=4096 * 64, ld_v=4096 * 64, ld_out=4096 * 64)
    assert lib.coral_lmhead_prompt_attention(ctypes.byref(big), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_TOO_LARGE


def _config(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_kv4_config), type=1, n_pages=10, page=32, n_heads=2, D=64, group=32)
    base.update(kw)
    return lmhead.coral_lmhead_kv4_config(**base)


CONFIG_BAD = [dict(struct_size=4), dict(type=0), dict(type=3), dict(n_pages=0), dict(page=0), dict(page=24), dict(page=-16), dict(n_heads=0),
              dict(n_heads=5000), dict(D=32), dict(D=96), dict(D=256), dict(group=16), dict(group=128), dict(group=0), dict(n_pages=2 ** 27)]


def _attention(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_kv4_attention_args), n_seq=2, n_rows=4, max_q=2, n_q=4, width=3, scale=0.125, ld_q=256,
                ld_out=256, ld_table=3, q_dev=P, table_dev=P, lens_dev=P, out_dev=P)
    base.update(kw)
    return lmhead.coral_lmhead_kv4_attention_args(**base)


@pytest.mark.parametrize("kw", CONFIG_BAD)
def test_kv4_bad_configurations(lib, kw):
    c, n, vp = _config(**kw), ctypes.c_size_t(), ctypes.c_void_p
    r = ctypes.byref(c)
    assert lib.coral_lmhead_kv4_bytes(r, ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_kv4_store(r, vp(P), vp(P), 1024, vp(P), 1024, vp(P), 1, None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_kv4_load(r, vp(P), vp(P), 1, vp(P), 1024, vp(P), 1024, None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_kv4_attention_bytes(r, ctypes.byref(_attention()), ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_kv4_attention(r, vp(P), ctypes.byref(_attention()), vp(P), None) == lmhead.CORAL_ERR_INVALID


def test_kv4_rows_refusals(lib):
    vp, r = ctypes.c_void_p, ctypes.byref(_config())
    store = lambda cache=P, k=P, ld_k=128, v=P, ld_v=128, slots=P, T=1: lib.coral_lmhead_kv4_store(r, vp(cache), vp(k), ld_k, vp(v), ld_v, vp(slots), T, None)
    load = lambda cache=P, k=P, ld_k=128, v=P, ld_v=128, slots=P, T=1: lib.coral_lmhead_kv4_load(r, vp(cache), vp(slots), T, vp(k), ld_k, vp(v), ld_v, None)
    for f in (store, load):
        for kw in (dict(cache=None), dict(cache=P + 16), dict(k=P + 8), dict(v=P + 2), dict(ld_k=120), dict(ld_v=132), dict(slots=None), dict(slots=P + 4), dict(T=-1)):
            assert f(**kw) == lmhead.CORAL_ERR_INVALID, kw
        assert f(T=2 ** 31 - 1) == lmhead.CORAL_ERR_TOO_LARGE
        assert f(T=0) == lmhead.CORAL_OK
    assert store(k=None) == lmhead.CORAL_ERR_INVALID and load(k=None, v=None) == lmhead.CORAL_ERR_INVALID
    n = ctypes.c_size_t()
    assert lib.coral_lmhead_kv4_bytes(r, ctypes.byref(n)) == 0 and n.value == 10 * 32 * 2 * (64 + 8 * 2)


@pytest.mark.parametrize("kw", [dict(struct_size=8), dict(n_seq=-1), dict(n_rows=-1), dict(max_q=0), dict(n_q=3), dict(n_q=0), dict(width=0), dict(ld_table=2),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(q_dev=None), dict(q_dev=P + 8), dict(out_dev=None), dict(table_dev=None),
                                dict(table_dev=P + 2), dict(lens_dev=None), dict(q_offsets_dev=P + 4), dict(tree_mask_dev=P + 4), dict(out_lse_dev=P + 2),
                                dict(ld_q=248), dict(ld_out=130), dict(max_q=65, n_rows=130, tree_mask_dev=P), dict(n_rows=3)])
def test_kv4_attention_refusals(lib, kw):
    n, r, a = ctypes.c_size_t(), ctypes.byref(_config()), _attention(**kw)
    assert lib.coral_lmhead_kv4_attention_bytes(r, ctypes.byref(a), ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_kv4_attention(r, ctypes.c_void_p(P), ctypes.byref(a), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID


def test_kv4_attention_refuses_bad_buffers_and_too_many_blocks(lib):
    vp, n, r, a = ctypes.c_void_p, ctypes.c_size_t(), ctypes.byref(_config()), _attention()
    for cache, ws in ((None, P), (P + 16, P), (P, None), (P, P + 16)):
        assert lib.coral_lmhead_kv4_attention(r, vp(cache), ctypes.byref(a), vp(ws), None) == lmhead.CORAL_ERR_INVALID
    big = _attention(n_seq=2 ** 20, n_rows=2 ** 30, max_q=1024, n_q=4)
    assert lib.coral_lmhead_kv4_attention_bytes(r, ctypes.byref(big), ctypes.byref(n)) == lmhead.CORAL_ERR_TOO_LARGE
    assert lib.coral_lmhead_kv4_attention_bytes(r, ctypes.byref(a), ctypes.byref(n)) == 0 and n.value >= 256
