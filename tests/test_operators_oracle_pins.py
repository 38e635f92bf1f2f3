"""The oracles of the 4-bit product and of the logits step on cases known by hand (CPU), and the refusals of both entry
points, which need no device."""
import ctypes

import numpy as np
import pytest

from oracle import operators_oracle as oor
from paper_2502_16880_b200 import build as cbuild
from paper_2502_16880_b200 import lmhead

P = 0x10000                                                # aligned, never dereferenced: each call below is refused


@pytest.fixture(scope="module")
def lib():
    cbuild.build_library()
    return lmhead.load_library()


def test_q4_by_hand():
    Wq = np.array([[0x21, 0x43], [0xF0, 0x88]], np.uint8)   # rows 1 2 3 4 and 0 15 8 8
    assert oor.q4_unpack(Wq).tolist() == [[1, 2, 3, 4], [0, 15, 8, 8]]
    x = np.array([[1.0, 10.0, 100.0, 1000.0]])
    out, size = oor.q4_linear(Wq, np.array([[2.0], [0.5]]), None, x)
    assert out.tolist() == [[2 * (-7 - 60 - 500 - 4000), 0.5 * (-8 + 70)]]
    assert size.tolist() == [[2 * 4567, 0.5 * 78]]
    out, _ = oor.q4_linear(Wq, np.array([[2.0, 3.0], [0.5, 1.0]]), np.array([[1, 4], [0, 8]]), x)
    assert out.tolist() == [[2 * 10 + 3 * (-100), 0.5 * 150]]


def test_logits_by_hand():
    l = [2.0, -2.0, 1.0, 0.0, 5.0]
    v, ids, lps, lse = oor.logits_row(l, 5, 3, prompt=[0, 1, 99, -1], output=[2, 2, 2], rep=2.0, freq=0.25, pres=1.0,
                                      bias=[(3, 1.0), (3, 4.0), (7, 9.0)], mask=[0b01111])
    assert v.tolist() == [1.0, -4.0, 0.5 - 0.75 - 1.0, 4.0, -np.inf]
    assert ids.tolist() == [3, 0, 2]
    assert np.isclose(np.exp([4.0, 1.0, -1.25, -4.0] - lse).sum(), 1.0) and np.allclose(lps, np.array([4.0, 1.0, -1.25]) - lse)
    v, ids, lps, lse = oor.logits_row(l, 5, 2, nothing=True)
    assert ids.tolist() == [oor.NO_TOKEN] * 2 and np.all(np.isneginf(lps)) and lse == -np.inf
    _, ids, _, _ = oor.logits_row([1.0, 3.0, 3.0, 1.0], 4, 3)
    assert ids.tolist() == [1, 2, 0]                        # equal values: the lower id


def _q4(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_q4_config), N=100, K=256, group=64, scale_type=1, has_zeros=0)
    base.update(kw)
    return lmhead.coral_lmhead_q4_config(**base)


@pytest.mark.parametrize("kw", [dict(struct_size=4), dict(N=0), dict(K=0), dict(K=32), dict(K=96), dict(group=16), dict(group=256),
                                dict(group=0), dict(scale_type=0), dict(scale_type=3), dict(has_zeros=2), dict(K=65536 + 64)])
def test_q4_bad_configurations(lib, kw):
    c, n = _q4(**kw), ctypes.c_size_t()
    vp = ctypes.c_void_p
    assert lib.coral_lmhead_q4_packed_bytes(ctypes.byref(c), ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_q4_pack(ctypes.byref(c), vp(P), vp(P), None, vp(P), None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_q4_linear(ctypes.byref(c), vp(P), vp(P), 1, 1, vp(P), 0, None, None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_q4_workspace_bytes(ctypes.byref(c), 1, ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID


def test_q4_bad_arguments(lib):
    c, vp = _q4(), ctypes.c_void_p
    cz = _q4(has_zeros=1)
    ok = [P, P, 1, 1, P, 0, None]
    for i, bad in [(0, None), (0, P + 128), (1, None), (1, P + 8), (2, 0), (2, 3), (3, 0), (3, -2), (4, None), (4, P + 2), (5, 3), (5, -1), (6, P + 64)]:
        a = list(ok)
        a[i] = bad
        assert lib.coral_lmhead_q4_linear(ctypes.byref(c), vp(a[0]), vp(a[1]), a[2], a[3], vp(a[4]), a[5], vp(a[6]), None) == \
            lmhead.CORAL_ERR_INVALID, (i, bad)
    for cfg, W, s, z, p in [(c, None, P, None, P), (c, P, None, None, P), (c, P, P, P, P), (cz, P, P, None, P), (c, P, P, None, None),
                            (c, P + 4, P, None, P), (c, P, P + 1, None, P), (c, P, P, None, P + 16)]:
        assert lib.coral_lmhead_q4_pack(ctypes.byref(cfg), vp(W), vp(s), vp(z), vp(p), None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_q4_linear(None, vp(P), vp(P), 1, 1, vp(P), 0, None, None) == lmhead.CORAL_ERR_INVALID
    assert lmhead.coral_lmhead_q4_workspace_bytes(c, 1) == 0 and lmhead.coral_lmhead_q4_workspace_bytes(c, 60) > 60 * 256 * 2
    for M in (17, 64, 1000):                               # a call that needs scratch and gets none
        assert lib.coral_lmhead_q4_linear(ctypes.byref(c), vp(P), vp(P), 1, M, vp(P), 0, None, None) == lmhead.CORAL_ERR_INVALID
    # sizes: 7 tiles of 16 rows x 2 blocks of 128 columns x (1024 + 16 rows x 2 groups x 2 or 4 bytes)
    assert lmhead.coral_lmhead_q4_packed_bytes(c) == 14 * (1024 + 64)
    assert lmhead.coral_lmhead_q4_packed_bytes(cz) == 14 * (1024 + 128)


def _largs(**kw):
    base = dict(struct_size=ctypes.sizeof(lmhead.coral_lmhead_logits_args), type=0, M=2, V=100, n_seq=2, k_tokens=5, ld_logits=100,
                ld_out=100, logits_dev=P, out_ids_dev=P, out_logprobs_dev=P, out_lse_dev=P)
    base.update(kw)
    return lmhead.coral_lmhead_logits_args(**base)


@pytest.mark.parametrize("kw", [
    dict(struct_size=16), dict(type=3), dict(type=-1), dict(M=0), dict(V=0), dict(V=(1 << 30) + 1, ld_logits=1 << 31), dict(logits_dev=None),
    dict(ld_logits=99), dict(out_logits_dev=P + 64, ld_out=99), dict(out_logits_dev=P, ld_out=101), dict(n_seq=1), dict(n_seq=-1),
    dict(k_tokens=33), dict(k_tokens=-1), dict(V=4, ld_logits=4), dict(out_ids_dev=None), dict(out_logprobs_dev=None),
    dict(k_tokens=0), dict(k_tokens=0, out_ids_dev=None, out_logprobs_dev=None, out_lse_dev=None),
    dict(prompt_tokens_dev=P), dict(prompt_offsets_dev=P), dict(output_tokens_dev=P), dict(output_offsets_dev=P),
    dict(prompt_tokens_dev=P, prompt_offsets_dev=P, prompt_total=-1), dict(prompt_tokens_dev=P, prompt_offsets_dev=P + 4),
    dict(output_tokens_dev=P + 2, output_offsets_dev=P), dict(output_tokens_dev=P, output_offsets_dev=P, output_total=1 << 31),
    dict(bias_tokens_dev=P), dict(bias_tokens_dev=P, bias_offsets_dev=P), dict(bias_values_dev=P),
    dict(bias_tokens_dev=P, bias_offsets_dev=P, bias_values_dev=P, bias_total=-1),
    dict(path_tokens_dev=P), dict(path_len=3), dict(path_len=-1), dict(path_tokens_dev=P, path_len=65), dict(mask_words_dev=P), dict(mask_rows_dev=P),
    dict(mask_words_dev=P, n_masks=1), dict(mask_words_dev=P, n_masks=0, mask_rows_dev=P), dict(logits_dev=P + 2),
    dict(type=1, logits_dev=P + 1), dict(repetition_dev=P + 1), dict(out_lse_dev=P + 2), dict(row_seq_dev=P + 1)])
def test_logits_refusals(lib, kw):
    a, n = _largs(**kw), ctypes.c_size_t()
    assert lib.coral_lmhead_logits_process(ctypes.byref(a), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID
    assert lib.coral_lmhead_logits_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == lmhead.CORAL_ERR_INVALID


def test_logits_refuses_null_workspaces_and_too_large_calls(lib):
    n = ctypes.c_size_t()
    assert lib.coral_lmhead_logits_process(None, ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_INVALID
    for ws in (None, P + 128):
        assert lib.coral_lmhead_logits_process(ctypes.byref(_largs()), ctypes.c_void_p(ws), None) == lmhead.CORAL_ERR_INVALID
    lists = dict(prompt_tokens_dev=P, prompt_offsets_dev=P, output_tokens_dev=P, output_offsets_dev=P, repetition_dev=P)
    for kw in (dict(M=1 << 30, V=1 << 20, ld_logits=1 << 20, n_seq=0), dict(prompt_total=1 << 30, output_total=1 << 30, **lists),
               dict(M=1, n_seq=1 << 29, **lists)):
        a = _largs(**kw)
        assert lib.coral_lmhead_logits_process(ctypes.byref(a), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_TOO_LARGE
    # lists cost two times four words (100 tokens) and a range a sequence and 8 + 4 bytes an element, rounded up to 256 bytes each
    size = lambda **kw: (lib.coral_lmhead_logits_workspace_bytes(ctypes.byref(_largs(**kw)), ctypes.byref(n)), n.value)[1]
    plain = size()
    assert size(prompt_total=100, output_total=50, **lists) == plain + 256 + 256 + 1280 + 768 + 256
    assert size(prompt_total=100, output_total=50, **{**lists, "repetition_dev": None}) == plain       # no penalty uses them


def test_q4_rows_of_a_pass_over_the_weights(lib):
    """The passes a call of up to 16 rows takes show in its workspace: behind the status word each has, rounded up to 256 bytes, an
    exponent a row, group sums and the rows themselves (rows of up to 1024 pieces of 8 columns are laid out in the kernel)."""
    up = lambda n: (n + 255) // 256 * 256
    for K, rows in ((4096, 16), (5632, 16), (8192, 11), (14336, 7), (28672, 3), (65536, 1)):
        c, KB = _q4(K=K, group=128), K // 128
        for M in (1, 2, 3, 7, 8, 11, 12, 16):
            parts = [min(rows, M - m) for m in range(0, M, rows)]
            want = sum(up(4 * r) + up(4 * r * KB) + up(256 * r * KB) for r in parts if r * KB * 16 > 1024)
            assert lmhead.coral_lmhead_q4_workspace_bytes(c, M) == (256 + want if want else 0), (K, M)


def test_q4_linear_asks_for_the_status_of_its_last_call(lib, monkeypatch):
    """Without a GPU: forward hands the library a workspace, status asks about that one, and calls that need none have status 0."""
    import torch
    calls, asked = [], []

    def status(workspace, stream=None):
        asked.append(workspace)
        return 0 if workspace is None else lmhead.CORAL_ERR_TIMEOUT

    monkeypatch.setattr(lmhead, "coral_lmhead_q4_pack", lambda *a: None)
    monkeypatch.setattr(lmhead, "coral_lmhead_q4_linear", lambda cfg, packed, x, out, workspace, stream: calls.append(workspace))
    monkeypatch.setattr(lmhead, "coral_lmhead_q4_status", status)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    lin = lmhead.Q4Linear(torch.zeros(48, 128, dtype=torch.uint8), torch.ones(48, 4, dtype=torch.bfloat16))
    assert lin.status() == 0 and asked == [None]
    for M in (33, 60):
        lin.forward(torch.zeros(M, 256, dtype=torch.bfloat16))
        assert calls[-1].numel() == lmhead.coral_lmhead_q4_workspace_bytes(lin.cfg, M)
        assert lin.status() == lmhead.CORAL_ERR_TIMEOUT and asked[-1] is calls[-1]
    lin.forward(torch.zeros(1, 256, dtype=torch.bfloat16))
    assert calls[-1] is None and lin.status() == 0


def test_logits_refuses_more_output_tokens_than_a_count_holds(lib):
    n = ctypes.c_size_t()
    lists = dict(output_tokens_dev=P, output_offsets_dev=P)
    most = (1 << 30) - 1
    size = lambda **kw: lib.coral_lmhead_logits_workspace_bytes(ctypes.byref(_largs(**lists, **kw)), ctypes.byref(n))
    assert size(frequency_dev=P, output_total=most) == 0
    assert size(frequency_dev=P, output_total=most + 1) == lmhead.CORAL_ERR_TOO_LARGE
    a = _largs(frequency_dev=P, output_total=most + 1, **lists)
    assert lib.coral_lmhead_logits_process(ctypes.byref(a), ctypes.c_void_p(P), None) == lmhead.CORAL_ERR_TOO_LARGE
    assert size(output_total=most + 1) == 0                  # no penalty: nothing is counted
