"""Thin ctypes binding of the C ABI in include/coral_lmhead.h.

Argument marshalling only: every step of the draft path runs in the CUDA
library.  torch is used for device memory and streams.  There is no CPU
fallback: if the compiled library is missing, loading fails with an error.
The function names are those of the C ABI; `LMHead` is a small convenience
wrapper that owns the device buffers.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# CORAL_LMHEAD_LIB selects another build of the same library (the range-checked one, see build.py)
LIB_PATH = os.environ.get("CORAL_LMHEAD_LIB") or os.path.join(_PKG, "libcoral_lmhead.so")

CORAL_OK = 0
CORAL_ERR_INVALID = -1
CORAL_ERR_GROUPING = -2
CORAL_ERR_CUDA = -3
CORAL_ERR_NOMEM = -4
CORAL_ERR_TIMEOUT = -5
CORAL_ERR_BOUNDS = -6
CORAL_ERR_TOO_LARGE = -7
CORAL_ERR_NONFINITE = -8
CORAL_ROUTE_STATIC_MAX_ROWS = 64
CORAL_OUTPUT_JOINT, CORAL_OUTPUT_FACTORISED, CORAL_OUTPUT_FACTORISED_RENORM = 0, 1, 2
CORAL_TYPE_F32, CORAL_TYPE_BF16, CORAL_TYPE_F16 = 0, 1, 2
CORAL_GATE_NONE, CORAL_GATE_CHANNEL, CORAL_GATE_ROW, CORAL_GATE_FULL = 0, 1, 2, 3
CORAL_PATH_AUTO, CORAL_PATH_STREAM, CORAL_PATH_TCGEN05, CORAL_PATH_SIMT_PLAIN, CORAL_PATH_ADAPTIVE = 0, 1, 2, 3, 4


class coral_lmhead_config(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("H", ctypes.c_int32), ("V", ctypes.c_int32),
                ("n_groups", ctypes.c_int32), ("max_M", ctypes.c_int32), ("max_k_groups", ctypes.c_int32),
                ("max_k_tokens", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class coral_lmhead_stats(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int32), ("M", ctypes.c_int32), ("k_groups", ctypes.c_int32),
                ("k_tokens", ctypes.c_int32), ("groups_touched", ctypes.c_int32),
                ("kernel_launches", ctypes.c_int32), ("weight_bytes", ctypes.c_int64),
                ("algorithmic_bytes", ctypes.c_int64)]


class coral_lmhead_norm_args(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("type", ctypes.c_int32), ("M", ctypes.c_int32), ("H", ctypes.c_int32),
                ("gate_mode", ctypes.c_int32), ("alpha", ctypes.c_float), ("eps", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("x_dev", "r_dev", "gate_dev", "w_post_dev", "w_pre_dev", "out_y_dev", "out_h_dev",
                                       "dy_dev", "dh_dev", "out_dx_dev", "out_dr_dev", "out_dgate_dev", "out_dw_pre_dev",
                                       "out_dw_post_dev")]


class coral_lmhead_q4_config(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("group", ctypes.c_int32),
                ("scale_type", ctypes.c_int32), ("has_zeros", ctypes.c_int32)]


class coral_lmhead_logits_args(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("type", "M", "V", "n_seq", "path_len", "n_masks", "k_tokens")] + [
        (n, ctypes.c_int64) for n in ("ld_logits", "ld_out", "prompt_total", "output_total", "bias_total")] + [
        (n, ctypes.c_void_p) for n in (
            "logits_dev", "out_logits_dev", "row_seq_dev", "prompt_tokens_dev", "output_tokens_dev", "path_tokens_dev",
            "bias_tokens_dev", "prompt_offsets_dev", "output_offsets_dev", "bias_offsets_dev", "repetition_dev",
            "frequency_dev", "presence_dev", "bias_values_dev", "mask_words_dev", "mask_rows_dev", "out_ids_dev",
            "out_logprobs_dev", "out_lse_dev")]


_lib = None
_vp, _i = ctypes.c_void_p, ctypes.c_int

_SIGNATURES = {
    "coral_lmhead_version": (_i, []),
    "coral_lmhead_query_sizes": (_i, [ctypes.POINTER(coral_lmhead_config), ctypes.POINTER(ctypes.c_size_t),
                                      ctypes.POINTER(ctypes.c_size_t)]),
    "coral_lmhead_create": (_i, [ctypes.POINTER(_vp), ctypes.POINTER(coral_lmhead_config), _vp, _vp, _vp, _vp, _vp, _vp]),
    "coral_lmhead_draft": (_i, [_vp, _vp, _i, _i, _i, _vp, _vp, _vp]),
    "coral_lmhead_draft_ex": (_i, [_vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "coral_lmhead_draft_host": (_i, [_vp, _vp, _i, _i, _i, _vp, _vp, _vp]),
    "coral_lmhead_set_group_shard": (_i, [_vp, _i, _i]),
    "coral_lmhead_draft_partial": (_i, [_vp, _vp, _i, _i, _i, _vp, _vp]),
    "coral_lmhead_merge_partials": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp]),
    "coral_lmhead_copy_floor": (_i, [_vp, ctypes.c_longlong, _i, _i, _vp]),
    "coral_lmhead_tc_issue_probe": (_i, [_vp, _i, _i, _i, _i, _vp, _vp]),
    "coral_lmhead_set_hot_groups": (_i, [_vp, _i]),
    "coral_csra_workspace_bytes": (_i, [_i, _i, _i, ctypes.POINTER(ctypes.c_size_t)]),
    "coral_csra_infonce": (_i, [_vp, _vp, _i, _i, _i, ctypes.c_float, _vp, _vp, _vp, _vp, _vp]),
    "coral_csra_status": (_i, [_vp, _vp]),
    "coral_lmhead_selftest_wait_expiry": (_i, [_vp, _vp]),
    "coral_lmhead_set_path": (_i, [_vp, _i]),
    "coral_lmhead_set_output_mode": (_i, [_vp, _i]),
    "coral_lmhead_set_router_mlp": (_i, [_vp, _vp, _vp]),
    "coral_lmhead_set_kernel_timing": (_i, [_vp, _i]),
    "coral_lmhead_head_kernel_ms": (_i, [_vp, ctypes.POINTER(ctypes.c_float)]),
    "coral_lmhead_stage_ms": (_i, [_vp] + [ctypes.POINTER(ctypes.c_float)] * 3),
    "coral_lmhead_status": (_i, [_vp, _vp]),
    "coral_lmhead_last_stats": (_i, [_vp, ctypes.POINTER(coral_lmhead_stats), _vp]),
    "coral_lmhead_route_static": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp]),
    "coral_tree_expand": (_i, [_vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "coral_lmhead_block_norm": (_i, [ctypes.POINTER(coral_lmhead_norm_args), _vp]),
    "coral_lmhead_block_norm_backward_bytes": (_i, [_i, _i, ctypes.POINTER(ctypes.c_size_t)]),
    "coral_lmhead_block_norm_backward": (_i, [ctypes.POINTER(coral_lmhead_norm_args), _vp, _vp]),
    "coral_lmhead_q4_packed_bytes": (_i, [ctypes.POINTER(coral_lmhead_q4_config), ctypes.POINTER(ctypes.c_size_t)]),
    "coral_lmhead_q4_pack": (_i, [ctypes.POINTER(coral_lmhead_q4_config), _vp, _vp, _vp, _vp, _vp]),
    "coral_lmhead_q4_workspace_bytes": (_i, [ctypes.POINTER(coral_lmhead_q4_config), _i, ctypes.POINTER(ctypes.c_size_t)]),
    "coral_lmhead_q4_linear": (_i, [ctypes.POINTER(coral_lmhead_q4_config), _vp, _vp, _i, _i, _vp, _i, _vp, _vp]),
    "coral_lmhead_q4_status": (_i, [_vp, _vp]),
    "coral_lmhead_logits_workspace_bytes": (_i, [ctypes.POINTER(coral_lmhead_logits_args), ctypes.POINTER(ctypes.c_size_t)]),
    "coral_lmhead_logits_process": (_i, [ctypes.POINTER(coral_lmhead_logits_args), _vp, _vp]),
    "coral_lmhead_error_string": (ctypes.c_char_p, [_i]),
    "coral_lmhead_destroy": (_i, [_vp]),
}


def load_library(path: str = LIB_PATH):
    """Load the compiled CUDA library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2502_16880_b200.build` "
                "(nvcc, sm_100a). There is no fallback path.")
        lib = ctypes.CDLL(path)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


class CoralError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {coral_lmhead_error_string(code)} ({code})")


def _check(code: int, where: str) -> None:
    if code != CORAL_OK:
        raise CoralError(code, where)


def _dev_ptr(t, dtype=None, allow_none=True):
    if t is None:
        if allow_none:
            return None
        raise ValueError("tensor required")
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _stream_ptr(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def make_config(H, V, n_groups, max_M, max_k_groups, max_k_tokens, shard=None) -> coral_lmhead_config:
    """shard = (rank, world): the handle stores and computes only the groups n with n % world == rank."""
    flags = 0 if shard is None else (int(shard[1]) & 0xFF) | ((int(shard[0]) & 0xFF) << 8)
    return coral_lmhead_config(ctypes.sizeof(coral_lmhead_config), H, V, n_groups, max_M, max_k_groups,
                               max_k_tokens, flags)


# ---- functions named as in the C ABI -------------------------------------------------
def coral_lmhead_version() -> int:
    return int(load_library().coral_lmhead_version())


def coral_lmhead_error_string(code: int) -> str:
    return load_library().coral_lmhead_error_string(int(code)).decode()


def coral_lmhead_query_sizes(cfg: coral_lmhead_config):
    pb, wb = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().coral_lmhead_query_sizes(ctypes.byref(cfg), ctypes.byref(pb), ctypes.byref(wb)),
           "coral_lmhead_query_sizes")
    return int(pb.value), int(wb.value)


def coral_lmhead_create(cfg, W_vocab, group_map_host, W_gate, packed_buf=None, workspace=None, stream=None):
    """W_vocab/W_gate: CUDA bf16 tensors; group_map_host: CPU int32 tensor [V]. Returns an opaque handle."""
    if group_map_host.is_cuda or group_map_host.dtype != torch.int32 or not group_map_host.is_contiguous():
        raise ValueError("group_map_host must be a contiguous CPU int32 tensor")
    if group_map_host.numel() != cfg.V:
        raise ValueError("group_map_host must have V entries")
    h = ctypes.c_void_p()
    _check(load_library().coral_lmhead_create(
        ctypes.byref(h), ctypes.byref(cfg), _dev_ptr(W_vocab, torch.bfloat16, False),
        ctypes.c_void_p(group_map_host.data_ptr()), _dev_ptr(W_gate, torch.bfloat16, False),
        _dev_ptr(packed_buf), _dev_ptr(workspace), _stream_ptr(stream)), "coral_lmhead_create")
    return h


def coral_lmhead_draft(handle, hidden, k_groups, k_tokens, out_ids, out_logprobs, stream=None):
    M = hidden.shape[0]
    _check(load_library().coral_lmhead_draft(
        handle, _dev_ptr(hidden, torch.bfloat16, False), M, int(k_groups), int(k_tokens),
        _dev_ptr(out_ids, torch.int32, False), _dev_ptr(out_logprobs, torch.float32, False), _stream_ptr(stream)),
        "coral_lmhead_draft")


def coral_lmhead_draft_ex(handle, hidden, k_groups, k_tokens, out_ids, out_logprobs, forced_groups=None,
                          out_groups=None, out_gate=None, out_logits=None, out_lse=None, stream=None):
    M = hidden.shape[0]
    _check(load_library().coral_lmhead_draft_ex(
        handle, _dev_ptr(hidden, torch.bfloat16, False), M, int(k_groups), int(k_tokens),
        _dev_ptr(forced_groups, torch.int32), _dev_ptr(out_groups, torch.int32), _dev_ptr(out_gate, torch.float32),
        _dev_ptr(out_logits, torch.float32), _dev_ptr(out_lse, torch.float32),
        _dev_ptr(out_ids, torch.int32, False), _dev_ptr(out_logprobs, torch.float32, False), _stream_ptr(stream)),
        "coral_lmhead_draft_ex")


def coral_lmhead_draft_host(handle, hidden_host, k_groups, k_tokens, out_ids_host, out_logprobs_host, stream=None):
    """Host (ideally pinned) buffers in and out; returns after the results are in host memory."""
    for t in (hidden_host, out_ids_host, out_logprobs_host):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("expected contiguous CPU tensors")
    M = hidden_host.shape[0]
    _check(load_library().coral_lmhead_draft_host(
        handle, ctypes.c_void_p(hidden_host.data_ptr()), M, int(k_groups), int(k_tokens),
        ctypes.c_void_p(out_ids_host.data_ptr()), ctypes.c_void_p(out_logprobs_host.data_ptr()),
        _stream_ptr(stream)), "coral_lmhead_draft_host")


def coral_lmhead_set_group_shard(handle, rank: int, world: int) -> None:
    _check(load_library().coral_lmhead_set_group_shard(handle, int(rank), int(world)), "coral_lmhead_set_group_shard")


def coral_lmhead_draft_partial(handle, hidden, k_groups, k_tokens, out_records, stream=None):
    """out_records: CUDA int32 tensor [M, 2 + 2 * k_tokens] (the per-row record of this GPU's groups)."""
    M = hidden.shape[0]
    if out_records.numel() != M * (2 + 2 * int(k_tokens)):
        raise ValueError("out_records must hold M x (2 + 2 k_tokens) words")
    _check(load_library().coral_lmhead_draft_partial(
        handle, _dev_ptr(hidden, torch.bfloat16, False), M, int(k_groups), int(k_tokens),
        _dev_ptr(out_records, torch.int32, False), _stream_ptr(stream)), "coral_lmhead_draft_partial")


def coral_lmhead_merge_partials(records, k_tokens, out_ids, out_logprobs, stream=None):
    """records: CUDA int32 tensor [world, M, 2 + 2 * k_tokens], rank-major as an all-gather leaves it."""
    world, M = records.shape[0], records.shape[1]
    _check(load_library().coral_lmhead_merge_partials(
        _dev_ptr(records, torch.int32, False), world, M, int(k_tokens), _dev_ptr(out_ids, torch.int32, False),
        _dev_ptr(out_logprobs, torch.float32, False), _stream_ptr(stream)), "coral_lmhead_merge_partials")


def draft_vocab_sharded(handle, hidden, k_groups, k_tokens, out_ids, out_logprobs, group=None, records=None,
                        gathered=None):
    """One vocab-sharded draft step on this rank of `group` (torch.distributed): this GPU's record per row,
    one all-gather of the records, the merge.  The handle must have been given this rank's shard with
    coral_lmhead_set_group_shard.  `records` [M, W] and `gathered` [world, M, W] (W = 2 + 2 k_tokens, int32)
    may be passed in to avoid allocating per call."""
    import torch.distributed as dist
    world = dist.get_world_size(group)
    M, W = hidden.shape[0], 2 + 2 * int(k_tokens)
    if records is None:
        records = torch.empty((M, W), dtype=torch.int32, device=hidden.device)
    if gathered is None:
        gathered = torch.empty((world, M, W), dtype=torch.int32, device=hidden.device)
    coral_lmhead_draft_partial(handle, hidden, k_groups, k_tokens, records)
    dist.all_gather_into_tensor(gathered.view(world * M, W), records.view(M, W), group=group)   # rank-major rows
    coral_lmhead_merge_partials(gathered, k_tokens, out_ids, out_logprobs)


def coral_lmhead_set_output_mode(handle, mode: int) -> None:
    _check(load_library().coral_lmhead_set_output_mode(handle, int(mode)), "coral_lmhead_set_output_mode")


def coral_lmhead_set_router_mlp(handle, W1=None, stream=None) -> None:
    """W1: CUDA bf16 [H, H] tensor of Eq. 7's first router layer, or None for the single-matrix gate."""
    _check(load_library().coral_lmhead_set_router_mlp(handle, _dev_ptr(W1, torch.bfloat16), _stream_ptr(stream)),
           "coral_lmhead_set_router_mlp")


def coral_lmhead_copy_floor(handle, nbytes: int, stream=None, in_flight: int = 0, repeats: int = 1) -> None:
    """Measurement aid: a do-nothing stream of the first `nbytes` of the packed head, `repeats` sweeps with
    `in_flight` 16 KiB copies outstanding per SM (0 = default); time it with events."""
    _check(load_library().coral_lmhead_copy_floor(handle, int(nbytes), int(in_flight), int(repeats),
                                                  _stream_ptr(stream)), "coral_lmhead_copy_floor")


def coral_lmhead_tc_issue_probe(handle, n: int, per_commit: int, issuers: int, rounds: int, out_ns, stream=None) -> None:
    """out_ns: CUDA int64 tensor of two words (issue time, completion time in ns of the first pair's first issuer)."""
    _check(load_library().coral_lmhead_tc_issue_probe(handle, int(n), int(per_commit), int(issuers), int(rounds),
                                                      _dev_ptr(out_ns, torch.int64, allow_none=False),
                                                      _stream_ptr(stream)), "coral_lmhead_tc_issue_probe")


def coral_csra_workspace_bytes(n: int, views: int, D: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().coral_csra_workspace_bytes(int(n), int(views), int(D), ctypes.byref(b)), "coral_csra_workspace_bytes")
    return int(b.value)


def coral_csra_infonce(Q, K, views, tau, workspace, out_loss, out_row_loss=None, out_logits=None, stream=None):
    """Q [n, D], K [views * n, D] CUDA bf16; workspace: CUDA uint8 tensor of coral_csra_workspace_bytes(n, views, D);
    out_loss [1] f32, out_row_loss [n] f32 or None, out_logits [n, views * n] f32 or None."""
    n, D = Q.shape
    if K.shape[0] != int(views) * n or K.shape[1] != D:
        raise ValueError("K must be [views * n, D]")
    _check(load_library().coral_csra_infonce(
        _dev_ptr(Q, torch.bfloat16, False), _dev_ptr(K, torch.bfloat16, False), n, int(views), D, float(tau),
        _dev_ptr(workspace, torch.uint8, False), _dev_ptr(out_row_loss, torch.float32),
        _dev_ptr(out_loss, torch.float32, False), _dev_ptr(out_logits, torch.float32), _stream_ptr(stream)),
        "coral_csra_infonce")


def coral_csra_status(workspace, stream=None) -> int:
    return int(load_library().coral_csra_status(_dev_ptr(workspace, torch.uint8, False), _stream_ptr(stream)))


def coral_lmhead_set_hot_groups(handle, n_hot: int) -> None:
    _check(load_library().coral_lmhead_set_hot_groups(handle, int(n_hot)), "coral_lmhead_set_hot_groups")


def coral_lmhead_selftest_wait_expiry(handle, stream=None) -> None:
    """Runs the kernels' bounded wait on a barrier nothing completes; coral_lmhead_status then reports a timeout."""
    _check(load_library().coral_lmhead_selftest_wait_expiry(handle, _stream_ptr(stream)),
           "coral_lmhead_selftest_wait_expiry")


def coral_lmhead_set_path(handle, path: int) -> None:
    _check(load_library().coral_lmhead_set_path(handle, int(path)), "coral_lmhead_set_path")


def coral_lmhead_set_kernel_timing(handle, on: bool) -> None:
    _check(load_library().coral_lmhead_set_kernel_timing(handle, int(bool(on))), "coral_lmhead_set_kernel_timing")


def coral_lmhead_head_kernel_ms(handle) -> float:
    ms = ctypes.c_float(0.0)
    _check(load_library().coral_lmhead_head_kernel_ms(handle, ctypes.byref(ms)), "coral_lmhead_head_kernel_ms")
    return float(ms.value)


def coral_lmhead_stage_ms(handle):
    """(route_ms, head_ms, merge_ms) of the last call made with kernel timing on."""
    a, b, c = ctypes.c_float(0.0), ctypes.c_float(0.0), ctypes.c_float(0.0)
    _check(load_library().coral_lmhead_stage_ms(handle, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
           "coral_lmhead_stage_ms")
    return float(a.value), float(b.value), float(c.value)


def coral_lmhead_status(handle, stream=None) -> int:
    return int(load_library().coral_lmhead_status(handle, _stream_ptr(stream)))


def coral_lmhead_last_stats(handle, stream=None) -> coral_lmhead_stats:
    s = coral_lmhead_stats()
    _check(load_library().coral_lmhead_last_stats(handle, ctypes.byref(s), _stream_ptr(stream)),
           "coral_lmhead_last_stats")
    return s


def coral_lmhead_route_static(W_gate, hidden, k_groups, out_groups, out_gate=None, stream=None) -> None:
    """Gate scores and top-k groups without a handle and without any allocation inside the library
    (for callers that are not allowed to allocate device memory); at most CORAL_ROUTE_STATIC_MAX_ROWS rows.
    The tensors passed in are the only memory the caller provides; scratch is built into the library."""
    N, H = W_gate.shape
    M = hidden.shape[0]
    _check(load_library().coral_lmhead_route_static(
        _dev_ptr(W_gate, torch.bfloat16, False), _dev_ptr(hidden, torch.bfloat16, False), M, H, N, int(k_groups),
        _dev_ptr(out_groups, torch.int32, False), _dev_ptr(out_gate, torch.float32), _stream_ptr(stream)),
        "coral_lmhead_route_static")


def coral_tree_expand(parent_scores, cand_ids, cand_logprobs, K, out_parent, out_token, out_score, stream=None):
    """parent_scores [n_seq, nodes] f32; cand_ids / cand_logprobs [n_seq, nodes, k_tokens] (or None); outputs [n_seq, K]."""
    n_seq, nodes = parent_scores.shape
    k_tokens = 1 if cand_logprobs is None else cand_logprobs.shape[-1]
    _check(load_library().coral_tree_expand(
        _dev_ptr(parent_scores, torch.float32, False), _dev_ptr(cand_ids, torch.int32), _dev_ptr(cand_logprobs, torch.float32),
        n_seq, nodes, k_tokens, int(K), _dev_ptr(out_parent, torch.int32, False), _dev_ptr(out_token, torch.int32, False),
        _dev_ptr(out_score, torch.float32, False), _stream_ptr(stream)), "coral_tree_expand")


# The operators around the draft step are called once per layer or token, so their checks are kept short: one line per
# tensor that returns its pointer, and the reason is looked for only when it fails.
_TYPES = {torch.float32: CORAL_TYPE_F32, torch.bfloat16: CORAL_TYPE_BF16, torch.float16: CORAL_TYPE_F16}


def _type_of(t) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"expected float32, bfloat16 or float16, got {t.dtype}")
    return _TYPES[t.dtype]


def _op_ptr(name, t, dtype, shape, dev):
    """Pointer of an operator's tensor (None stays None) of this type and shape, contiguous, on device index `dev`: the
    library launches on the current device and reads and writes as many elements as the other arguments say."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{dev}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    raise ValueError(f"{name}: expected {dtype} {shape if shape is not None else ''}, got {t.dtype} {tuple(t.shape)}")


def _op_device(t, name) -> int:
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current CUDA device")
    return dev


def _op_stream(stream, dev) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _op_scratch(n, device, stream):
    """Scratch of one call, of the pool of the stream that runs it: what had the memory before and what gets it next run on
    that stream too, before and behind the call."""
    if stream is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=torch.uint8, device=device)


def _op_output(shape, dtype, device, stream):
    """A result that `stream` writes and the caller's current stream reads: of the pool of the former, like scratch, and given
    back only when what the latter has been asked to do by then is done."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        out = torch.empty(shape, dtype=dtype, device=device)
    out.record_stream(torch.cuda.current_stream(device))
    return out


_NORM_SIZE = ctypes.sizeof(coral_lmhead_norm_args)


def _norm_args(x, r, w_pre, eps, w_post, gate, gate_mode, alpha, dev, out_y=None, out_h=None, dy=None, dh=None, out_dx=None,
               out_dr=None, out_dgate=None, out_dw_pre=None, out_dw_post=None):
    if x.dim() != 2:
        raise ValueError("x must be [M, H]")
    shape, t, f = x.shape, x.dtype, torch.float32
    M, H = shape
    g_shape = None if gate is None else (H,) if gate_mode == CORAL_GATE_CHANNEL else (M,) if gate_mode == CORAL_GATE_ROW else shape
    return coral_lmhead_norm_args(
        _NORM_SIZE, _type_of(x), M, H, gate_mode, alpha, eps, _op_ptr("x", x, t, shape, dev), _op_ptr("r", r, t, shape, dev),
        _op_ptr("gate", gate, t, g_shape, dev), _op_ptr("w_post", w_post, t, (H,), dev), _op_ptr("w_pre", w_pre, t, (H,), dev),
        _op_ptr("out_y", out_y, t, shape, dev), _op_ptr("out_h", out_h, t, shape, dev), _op_ptr("dy", dy, t, shape, dev),
        _op_ptr("dh", dh, t, shape, dev), _op_ptr("out_dx", out_dx, t, shape, dev), _op_ptr("out_dr", out_dr, t, shape, dev),
        _op_ptr("out_dgate", out_dgate, t if gate_mode == CORAL_GATE_FULL else f, g_shape, dev),
        _op_ptr("out_dw_pre", out_dw_pre, f, (H,), dev), _op_ptr("out_dw_post", out_dw_post, f, (H,), dev))


def coral_lmhead_block_norm(x, r, w_pre, eps, out_y, out_h, w_post=None, gate=None, gate_mode=CORAL_GATE_NONE, alpha=1.0,
                            stream=None):
    """y = alpha r + gate b with b = x, or its norm times w_post; h = the norm of y times w_pre.  x, r, out_y, out_h:
    [M, H]; gate: [H], [M] or [M, H] by gate_mode (CORAL_GATE_*).  r, w_pre with out_h, or out_y may be None."""
    dev = _op_device(x, "x")
    a = _norm_args(x, r, w_pre, eps, w_post, gate, gate_mode, alpha, dev, out_y, out_h)
    _check((_lib or load_library()).coral_lmhead_block_norm(ctypes.byref(a), _op_stream(stream, dev)), "coral_lmhead_block_norm")


def coral_lmhead_block_norm_backward_bytes(M: int, H: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().coral_lmhead_block_norm_backward_bytes(int(M), int(H), ctypes.byref(b)),
           "coral_lmhead_block_norm_backward_bytes")
    return int(b.value)


def coral_lmhead_block_norm_backward(x, r, w_pre, eps, dy, dh, workspace, out_dx, out_dr=None, out_dw_pre=None, w_post=None,
                                     gate=None, gate_mode=CORAL_GATE_NONE, alpha=1.0, out_dw_post=None, out_dgate=None,
                                     stream=None):
    """Gradient of coral_lmhead_block_norm.  dy, dh: gradients of y and h (one may be None); out_dx, out_dr like x;
    out_dw_pre, out_dw_post: fp32 [H]; out_dgate: fp32 [H] or [M], or like x for a full gate; workspace: CUDA uint8
    tensor of coral_lmhead_block_norm_backward_bytes(M, H)."""
    dev = _op_device(x, "x")
    a = _norm_args(x, r, w_pre, eps, w_post, gate, gate_mode, alpha, dev, None, None, dy, dh, out_dx, out_dr, out_dgate,
                   out_dw_pre, out_dw_post)
    if workspace.numel() < coral_lmhead_block_norm_backward_bytes(*x.shape):
        raise ValueError("workspace is smaller than coral_lmhead_block_norm_backward_bytes(M, H)")
    _check((_lib or load_library()).coral_lmhead_block_norm_backward(
        ctypes.byref(a), _op_ptr("workspace", workspace, torch.uint8, None, dev), _op_stream(stream, dev)),
        "coral_lmhead_block_norm_backward")


def make_q4_config(N, K, group, scale_dtype, has_zeros) -> coral_lmhead_q4_config:
    return coral_lmhead_q4_config(ctypes.sizeof(coral_lmhead_q4_config), int(N), int(K), int(group), _TYPES[scale_dtype],
                                  int(bool(has_zeros)))


def coral_lmhead_q4_packed_bytes(cfg: coral_lmhead_q4_config) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().coral_lmhead_q4_packed_bytes(ctypes.byref(cfg), ctypes.byref(b)), "coral_lmhead_q4_packed_bytes")
    return int(b.value)


def coral_lmhead_q4_pack(cfg, Wq, scales, zeros, packed, stream=None) -> None:
    """Wq: CUDA uint8 [N, K / 2], low four bits first; scales: bf16 or fp16 [N, K / group]; zeros: uint8 like scales, or
    None (8 everywhere); packed: CUDA uint8 tensor of coral_lmhead_q4_packed_bytes(cfg)."""
    dev = _op_device(Wq, "Wq")
    g = (cfg.N, cfg.K // cfg.group)
    sdt = torch.bfloat16 if cfg.scale_type == CORAL_TYPE_BF16 else torch.float16
    if packed.numel() < coral_lmhead_q4_packed_bytes(cfg):
        raise ValueError("packed is smaller than coral_lmhead_q4_packed_bytes(cfg)")
    _check(load_library().coral_lmhead_q4_pack(
        ctypes.byref(cfg), _op_ptr("Wq", Wq, torch.uint8, (cfg.N, cfg.K // 2), dev), _op_ptr("scales", scales, sdt, g, dev),
        _op_ptr("zeros", zeros, torch.uint8, g, dev), _op_ptr("packed", packed, torch.uint8, None, dev), _op_stream(stream, dev)),
        "coral_lmhead_q4_pack")


def coral_lmhead_q4_workspace_bytes(cfg, M: int) -> int:
    b = ctypes.c_size_t(0)
    _check((_lib or load_library()).coral_lmhead_q4_workspace_bytes(ctypes.byref(cfg), M, ctypes.byref(b)),
           "coral_lmhead_q4_workspace_bytes")
    return b.value


def coral_lmhead_q4_linear(cfg, packed, x, out, workspace=None, stream=None) -> None:
    """out [M, N] (fp32, bf16 or fp16) = x [M, K] (bf16 or fp16) times the packed weights' transpose.  workspace: CUDA uint8
    tensor of coral_lmhead_q4_workspace_bytes(cfg, M), None if that is 0."""
    dev = _op_device(x, "x")
    M, N, K, group = x.shape[0], cfg.N, cfg.K, cfg.group
    if packed.numel() < (N + 15) // 16 * ((K + 127) // 128) * (1024 + 2048 // group * (4 if cfg.has_zeros else 2)):
        raise ValueError("packed is smaller than coral_lmhead_q4_packed_bytes(cfg)")
    if workspace is not None and workspace.numel() < coral_lmhead_q4_workspace_bytes(cfg, M):
        raise ValueError("workspace is smaller than coral_lmhead_q4_workspace_bytes(cfg, M)")
    _check((_lib or load_library()).coral_lmhead_q4_linear(
        ctypes.byref(cfg), _op_ptr("packed", packed, torch.uint8, None, dev), _op_ptr("x", x, x.dtype, (M, K), dev),
        _type_of(x), M, _op_ptr("out", out, out.dtype, (M, N), dev), _type_of(out),
        _op_ptr("workspace", workspace, torch.uint8, None, dev), _op_stream(stream, dev)), "coral_lmhead_q4_linear")


def coral_lmhead_q4_status(workspace, stream=None) -> int:
    """Status word of the last call that used the workspace; waits for the stream."""
    return int((_lib or load_library()).coral_lmhead_q4_status(None if workspace is None else workspace.data_ptr(), _stream_ptr(stream)))


def _rows_ptr(name, t, dtype, shape, dev):
    """Pointer and row distance of a matrix whose rows may lie apart (a slice of padded rows)."""
    if t is None:
        return None, 0
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{dev}")
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    M, V = shape
    if t.is_contiguous():
        return t.data_ptr(), V
    ld = t.stride(0) if M > 1 else V
    if (V > 1 and t.stride(1) != 1) or ld < V:
        raise ValueError(f"{name}: the elements of a row must be contiguous and rows must not overlap")
    return t.data_ptr(), ld


def _list_ptrs(name, tokens, offsets, n_seq, dev):
    """Pointers and length of a flat token list and its offsets; lists that are all empty count as absent."""
    if tokens is None or offsets is None:
        if tokens is not offsets:
            raise ValueError(f"{name}_tokens and {name}_offsets go together")
        return None, None, 0
    n = tokens.numel()
    if n == 0:
        return None, None, 0
    return (_op_ptr(name + "_tokens", tokens, torch.int32, (n,), dev),
            _op_ptr(name + "_offsets", offsets, torch.int64, (n_seq + 1,), dev), n)


_LOGITS_SIZE = ctypes.sizeof(coral_lmhead_logits_args)


def coral_lmhead_logits_process(logits, *, row_seq=None, prompt_tokens=None, prompt_offsets=None, output_tokens=None,
                                output_offsets=None, path_tokens=None, repetition=None, frequency=None, presence=None,
                                bias_tokens=None, bias_values=None, bias_offsets=None, mask_words=None, mask_rows=None,
                                out_logits=None, out_ids=None, out_logprobs=None, out_lse=None, stream=None) -> None:
    """Penalties, biases and masks on logits [M, V] (rows may lie apart), and the candidates of the result.  Lists are flat
    int32 with int64 offsets [n_seq + 1]; path_tokens int32 [M, path_len]; repetition, frequency, presence fp32 [n_seq];
    mask_words int32 [n_masks, ceil(V / 32)]; out_ids int32 and out_logprobs fp32 [M, k_tokens]; out_lse fp32 [M].  The scratch
    of the call comes from torch's allocator."""
    dev = _op_device(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must be [M, V]")
    shape, t = logits.shape, logits.dtype
    M, V = shape
    i32, f32 = torch.int32, torch.float32
    n_seq = 0                                        # no lists and no penalties: no sequences
    for p in (repetition, frequency, presence):
        if p is not None:
            n_seq = p.numel()
            break
    else:
        for o in (prompt_offsets, output_offsets, bias_offsets):
            if o is not None:
                n_seq = o.numel() - 1
                break
    path_len = 0 if path_tokens is None else path_tokens.shape[1]
    n_masks = 0 if mask_words is None else mask_words.shape[0]
    k = 0 if out_ids is None else out_ids.shape[1]
    in_ptr, ld_in = _rows_ptr("logits", logits, t, shape, dev)
    out_ptr, ld_out = _rows_ptr("out_logits", out_logits, t, shape, dev)
    prompt, prompt_off, prompt_n = _list_ptrs("prompt", prompt_tokens, prompt_offsets, n_seq, dev)
    output, output_off, output_n = _list_ptrs("output", output_tokens, output_offsets, n_seq, dev)
    bias, bias_off, bias_n = _list_ptrs("bias", bias_tokens, bias_offsets, n_seq, dev)
    a = coral_lmhead_logits_args(
        _LOGITS_SIZE, _type_of(logits), M, V, n_seq, path_len, n_masks, k, ld_in, ld_out, prompt_n, output_n, bias_n, in_ptr,
        out_ptr, _op_ptr("row_seq", row_seq, i32, (M,), dev), prompt, output,
        _op_ptr("path_tokens", path_tokens, i32, (M, path_len), dev) if path_len else None, bias, prompt_off, output_off, bias_off,
        _op_ptr("repetition", repetition, f32, (n_seq,), dev), _op_ptr("frequency", frequency, f32, (n_seq,), dev),
        _op_ptr("presence", presence, f32, (n_seq,), dev), _op_ptr("bias_values", bias_values, f32, (bias_n,), dev) if bias_n else None,
        _op_ptr("mask_words", mask_words, i32, (n_masks, (V + 31) // 32), dev), _op_ptr("mask_rows", mask_rows, i32, (M,), dev),
        _op_ptr("out_ids", out_ids, i32, (M, k), dev), _op_ptr("out_logprobs", out_logprobs, f32, (M, k), dev),
        _op_ptr("out_lse", out_lse, f32, (M,), dev))
    lib, n = _lib or load_library(), ctypes.c_size_t(0)
    _check(lib.coral_lmhead_logits_workspace_bytes(ctypes.byref(a), ctypes.byref(n)), "coral_lmhead_logits_workspace_bytes")
    workspace = _op_scratch(n.value, logits.device, stream)
    _check(lib.coral_lmhead_logits_process(ctypes.byref(a), workspace.data_ptr(), _op_stream(stream, dev)),
           "coral_lmhead_logits_process")


def coral_lmhead_destroy(handle) -> None:
    _check(load_library().coral_lmhead_destroy(handle), "coral_lmhead_destroy")


# ---- convenience wrapper ---------------------------------------------------------------
class LMHead:
    """Owns the packed weights and workspace (torch allocations) of one handle."""

    def __init__(self, W_vocab, group_map_host, W_gate, max_M, max_k_groups, max_k_tokens=10, shard=None):
        V, H = W_vocab.shape
        N = W_gate.shape[0]
        self.cfg = make_config(H, V, N, max_M, max_k_groups, max_k_tokens, shard)
        pb, wb = coral_lmhead_query_sizes(self.cfg)
        dev = W_vocab.device
        self.packed = torch.empty(pb, dtype=torch.uint8, device=dev)
        self.workspace = torch.empty(wb, dtype=torch.uint8, device=dev)
        self.handle = coral_lmhead_create(self.cfg, W_vocab, group_map_host, W_gate, self.packed, self.workspace)
        self.device = dev

    def draft(self, hidden, k_groups, k_tokens, taps=False, forced_groups=None, stream=None):
        M = hidden.shape[0]
        dev = self.device
        ids = torch.empty((M, k_tokens), dtype=torch.int32, device=dev)
        lps = torch.empty((M, k_tokens), dtype=torch.float32, device=dev)
        if not taps and forced_groups is None:
            coral_lmhead_draft(self.handle, hidden, k_groups, k_tokens, ids, lps, stream)
            return ids, lps
        v = self.cfg.V // self.cfg.n_groups
        out = {
            "groups": torch.empty((M, k_groups), dtype=torch.int32, device=dev),
            "gate": torch.empty((M, self.cfg.n_groups), dtype=torch.float32, device=dev),
            "logits": torch.empty((M, k_groups, v), dtype=torch.float32, device=dev),
            "lse": torch.empty((M,), dtype=torch.float32, device=dev),
        }
        coral_lmhead_draft_ex(self.handle, hidden, k_groups, k_tokens, ids, lps, forced_groups=forced_groups,
                              out_groups=out["groups"], out_gate=out["gate"], out_logits=out["logits"],
                              out_lse=out["lse"], stream=stream)
        out["ids"], out["logprobs"] = ids, lps
        return out

    def set_path(self, path):
        coral_lmhead_set_path(self.handle, path)

    def status(self):
        return coral_lmhead_status(self.handle)

    def stats(self):
        return coral_lmhead_last_stats(self.handle)

    def close(self):
        if self.handle is not None:
            coral_lmhead_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Q4Linear:
    """Owns the packed copy of one 4-bit weight matrix: Wq uint8 [N, K / 2], scales [N, K / group] (bf16 or fp16), zeros
    uint8 like scales or None.  The inputs may be freed after construction."""

    def __init__(self, Wq, scales, zeros=None):
        N, K = Wq.shape[0], 2 * Wq.shape[1]
        if scales.dim() != 2 or scales.shape[1] < 1 or K % scales.shape[1]:
            raise ValueError("scales must be [N, K / group]")
        if scales.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("scales must be bfloat16 or float16")
        self.cfg = make_q4_config(N, K, K // scales.shape[1], scales.dtype, zeros is not None)
        self.packed = torch.empty(coral_lmhead_q4_packed_bytes(self.cfg), dtype=torch.uint8, device=Wq.device)
        self._workspace = None
        coral_lmhead_q4_pack(self.cfg, Wq, scales, zeros, self.packed)

    def forward(self, x, out=None, out_dtype=torch.float32, stream=None):
        """x [M, K] times the weights' transpose; the scratch of a call comes from torch's allocator, call by call, so calls
        on several streams do not share any.  That of the last call is kept for status()."""
        M = x.shape[0]
        if out is None:
            out = _op_output((M, self.cfg.N), out_dtype, x.device, stream)
        n = coral_lmhead_q4_workspace_bytes(self.cfg, M)
        self._workspace = workspace = _op_scratch(n, x.device, stream) if n else None
        coral_lmhead_q4_linear(self.cfg, self.packed, x, out, workspace, stream)
        return out

    def status(self, stream=None):
        """Status of the last forward (0, or CORAL_ERR_TIMEOUT: a bounded wait ran out and the results mean nothing); waits for
        `stream`, the one that ran it, or else for the device.  A forward captured into a graph has one once the graph has run."""
        if stream is None and self._workspace is not None:
            torch.cuda.synchronize(self._workspace.device)
        return coral_lmhead_q4_status(self._workspace, stream)
