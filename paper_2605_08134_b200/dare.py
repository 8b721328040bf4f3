"""ctypes binding of libdare: the same entry points as include/dare.h, argument marshalling only.

Every step of the path runs inside the CUDA library; torch is used by callers for device memory and streams.
Importing this module loads the shared library and fails loudly if it is missing (there is no fallback).
"""
from __future__ import annotations

import ctypes as C
import os
import struct

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdare.so")

OK = 0
ERR_INVALID_ARG, ERR_SHAPE, ERR_STATE, ERR_ALIGN, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED, \
    ERR_DEVICE_CHECK = range(1, 10)
MODE_DENSE, MODE_KV, MODE_O, MODE_BOTH = 0, 1, 2, 3
FORM_SCORE_FIRST, FORM_SPLIT_Q, FORM_SPLIT_KV, FORM_SPLIT_OUT = 1, 2, 4, 8
F32, BF16 = 0, 1
PATH_AUTO, PATH_SIMT, PATH_TENSOR = 0, 1, 2
ROPE_SCALE = {"none": 0, "linear": 1, "base": 2, "turns": 3, "index": 4}
ROPE_LAYOUT = {"half": 0, "interleaved": 1}
ACT = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


class LayerConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("d_model", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float),
                ("dtype", C.c_int32), ("score_head", C.c_int32), ("kernel_path", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [("w_q", C.c_void_p), ("w_k", C.c_void_p), ("w_v", C.c_void_p), ("w_o", C.c_void_p),
                ("rms_gain", C.c_void_p)]


class StackConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_int32), ("d_ff", C.c_int32), ("vocab", C.c_int32),
                ("mask_id", C.c_int32), ("block", C.c_int32), ("layer", LayerConfig)]


class BlockWeights(C.Structure):
    _fields_ = [("attn", LayerWeights), ("gain2", C.c_void_p), ("w_gate", C.c_void_p), ("w_up", C.c_void_p),
                ("w_down", C.c_void_p)]


class StackWeights(C.Structure):
    _fields_ = [("emb", C.c_void_p), ("head", C.c_void_p), ("final_gain", C.c_void_p),
                ("blocks_host", C.POINTER(BlockWeights))]


class RopeConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("rotary_dim", C.c_int32), ("theta", C.c_double), ("scaling", C.c_int32),
                ("trained", C.c_int32), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("magnitude", C.c_double)]


class RopeApply(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("tokens", C.c_int64), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("transpose", C.c_int32),
                ("pos_begin", C.c_int32), ("x_token", C.c_int64), ("x_head", C.c_int64), ("y_token", C.c_int64),
                ("y_head", C.c_int64), ("table_positions", C.c_int64)]


class LinearConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("rows", C.c_int64), ("in_features", C.c_int32),
                ("out_features", C.c_int32), ("activation", C.c_int32), ("reserved", C.c_int32), ("x_row", C.c_int64),
                ("w_row", C.c_int64), ("resid_row", C.c_int64), ("y_row", C.c_int64)]


class AttentionConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("batch", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float),
                ("q_rows", C.c_int64), ("k_rows", C.c_int64), ("q_token", C.c_int64), ("q_head", C.c_int64),
                ("k_token", C.c_int64), ("k_head", C.c_int64), ("v_token", C.c_int64), ("v_head", C.c_int64),
                ("o_token", C.c_int64), ("o_head", C.c_int64)]


class DareError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_08134_b200.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, f32, sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
    sig = {
        "dare_abi_version": (C.c_int, []),
        "dare_status_string": (C.c_char_p, [C.c_int]),
        "dare_layer_workspace_bytes": (sz, [C.POINTER(LayerConfig)]),
        "dare_layer_create": (C.c_int, [C.POINTER(LayerConfig), C.POINTER(LayerWeights), vp, sz, C.POINTER(vp)]),
        "dare_layer_step": (C.c_int, [vp, vp, i32, i32, i32, i32, f32, vp, vp]),
        "dare_layer_step_host": (C.c_int, [vp, vp, i32, i32, i32, i32, f32, vp, vp]),
        "dare_layer_step_host_async": (C.c_int, [vp, vp, i32, i32, i32, i32, f32, vp, vp]),
        "dare_layer_wait_host": (C.c_int, [vp]),
        "dare_layer_step_quantile": (C.c_int, [vp, vp, i32, i32, i32, i32, i32, vp, vp]),
        "dare_layer_last_threshold": (C.c_int, [vp, C.POINTER(C.c_float), vp]),
        "dare_score_kth": (C.c_int, [vp, C.c_int64, C.c_int64, vp, vp]),
        "dare_rmsnorm": (C.c_int, [vp, vp, vp, C.c_int64, i32, f32, i32, vp]),
        "dare_layer_reset": (C.c_int, [vp]),
        "dare_layer_destroy": (C.c_int, [vp]),
        "dare_layer_status": (C.c_int, [vp, vp]),
        "dare_layer_clear_status": (C.c_int, [vp, vp]),
        "dare_layer_debug_wait_probe": (C.c_int, [vp, C.c_uint64, C.POINTER(C.c_uint64), vp]),
        "dare_layer_debug_inject": (C.c_int, [vp, C.c_int]),
        "dare_layer_last_selection": (C.c_int, [vp, vp, vp, vp, vp, vp, vp]),
        "dare_layer_read_caches": (C.c_int, [vp, vp, vp, vp, vp, vp]),
        "dare_layer_state_bytes": (sz, [vp]),
        "dare_layer_export_state": (C.c_int, [vp, vp, sz, vp]),
        "dare_layer_import_state": (C.c_int, [vp, vp, sz, vp]),
        "dare_layer_last_launch_count": (C.c_int, [vp]),
        "dare_layer_last_forms": (C.c_int, [vp]),
        "dare_layer_set_profiling": (C.c_int, [vp, i32]),
        "dare_layer_last_kernel_times": (C.c_int, [vp, vp, vp, i32, C.POINTER(C.c_int)]),
        "dare_kernel_slot_name": (C.c_char_p, [C.c_int]),
        "dare_stack_workspace_bytes": (sz, [C.POINTER(StackConfig)]),
        "dare_stack_create": (C.c_int, [C.POINTER(StackConfig), C.POINTER(StackWeights), vp, sz, C.POINTER(vp)]),
        "dare_stack_reset": (C.c_int, [vp]),
        "dare_stack_destroy": (C.c_int, [vp]),
        "dare_stack_layer": (vp, [vp, i32]),
        "dare_stack_forward": (C.c_int, [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp]),
        "dare_stack_set_capture": (C.c_int, [vp, i32, vp, vp]),
        "dare_stack_last_hidden": (C.c_int, [vp, vp, sz, vp]),
        "dare_stack_decode_step": (C.c_int, [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]),
        "dare_layer_debug_timestamps": (C.c_int, [vp, i32, vp, vp]),
        "dare_drift_scores": (C.c_int, [vp, vp, C.c_int64, i32, vp, vp]),
        "dare_select_compact_scratch_bytes": (sz, [C.c_int64]),
        "dare_select_compact": (C.c_int, [vp, C.c_int64, f32, vp, vp, vp, sz, vp]),
        "dare_select_compact_static_max_tokens": (C.c_int64, []),
        "dare_select_compact_static": (C.c_int, [vp, C.c_int64, f32, vp, vp, vp]),
        "dare_rope_table": (C.c_int, [C.POINTER(RopeConfig), vp, C.c_int64, vp]),
        "dare_rope": (C.c_int, [C.POINTER(RopeApply), vp, vp, vp, vp, vp, vp]),
        "dare_linear": (C.c_int, [C.POINTER(LinearConfig), vp, vp, vp, vp, vp, vp, vp]),
        "dare_attention_workspace_bytes": (sz, [C.POINTER(AttentionConfig)]),
        "dare_attention": (C.c_int, [C.POINTER(AttentionConfig), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib, tuple(sig)


_lib, EXPORTS = _load()


def status_string(status: int) -> str:
    return _lib.dare_status_string(status).decode()


def abi_version() -> int:
    return _lib.dare_abi_version()


def make_config(d_model, n_heads, head_dim, max_batch, max_seq, rope_theta, rms_eps, dtype, score_head=0,
                kernel_path=PATH_AUTO) -> LayerConfig:
    return LayerConfig(C.sizeof(LayerConfig), d_model, n_heads, head_dim, max_batch, max_seq, rope_theta, rms_eps,
                       dtype, score_head, kernel_path)


def dare_layer_workspace_bytes(cfg: LayerConfig) -> int:
    return _lib.dare_layer_workspace_bytes(C.byref(cfg))


def dare_layer_create(cfg: LayerConfig, weights: LayerWeights, workspace_ptr: int, workspace_bytes: int):
    """-> (status, handle)"""
    out = C.c_void_p()
    st = _lib.dare_layer_create(C.byref(cfg) if cfg is not None else None,
                                C.byref(weights) if weights is not None else None,
                                workspace_ptr, workspace_bytes, C.byref(out))
    return st, out.value


def dare_layer_step(handle, x_ptr, batch, seq_act, pos_begin, mode, threshold, y_ptr, stream=0) -> int:
    return _lib.dare_layer_step(handle, x_ptr, batch, seq_act, pos_begin, mode, threshold, y_ptr, stream)


def dare_layer_step_host(handle, x_host_ptr, batch, seq_act, pos_begin, mode, threshold, y_host_ptr, stream=0) -> int:
    return _lib.dare_layer_step_host(handle, x_host_ptr, batch, seq_act, pos_begin, mode, threshold, y_host_ptr, stream)


def dare_layer_step_host_async(handle, x_host_ptr, batch, seq_act, pos_begin, mode, threshold, y_host_ptr, stream=0) -> int:
    return _lib.dare_layer_step_host_async(handle, x_host_ptr, batch, seq_act, pos_begin, mode, threshold, y_host_ptr,
                                           stream)


def dare_layer_wait_host(handle) -> int:
    return _lib.dare_layer_wait_host(handle)


def dare_layer_reset(handle) -> int:
    return _lib.dare_layer_reset(handle)


def dare_layer_destroy(handle) -> int:
    return _lib.dare_layer_destroy(handle)


def dare_layer_status(handle, stream=0) -> int:
    return _lib.dare_layer_status(handle, stream)


def dare_layer_step_quantile(handle, x_ptr, batch, seq_act, pos_begin, mode, reuse_count, y_ptr, stream=0) -> int:
    return _lib.dare_layer_step_quantile(handle, x_ptr, batch, seq_act, pos_begin, mode, reuse_count, y_ptr, stream)


def dare_layer_last_threshold(handle, stream=0):
    """-> (status, tau of the last step)."""
    tau = C.c_float(0.0)
    st = _lib.dare_layer_last_threshold(handle, C.byref(tau), stream)
    return st, float(tau.value)


def dare_rmsnorm(x_ptr, gain_ptr, y_ptr, rows, d_model, eps, dtype, stream=0) -> int:
    return _lib.dare_rmsnorm(x_ptr, gain_ptr, y_ptr, rows, d_model, eps, dtype, stream)


def dare_score_kth(scores_ptr, n_tokens, k, tau_out_ptr, stream=0) -> int:
    return _lib.dare_score_kth(scores_ptr, n_tokens, k, tau_out_ptr, stream)


def dare_layer_clear_status(handle, stream=0) -> int:
    return _lib.dare_layer_clear_status(handle, stream)


def dare_layer_debug_wait_probe(handle, limit_ns, stream=0):
    """-> (status, nanoseconds the probe's wait took before it gave up)."""
    waited = C.c_uint64(0)
    st = _lib.dare_layer_debug_wait_probe(handle, limit_ns, C.byref(waited), stream)
    return st, int(waited.value)


def dare_layer_debug_inject(handle, what) -> int:
    return _lib.dare_layer_debug_inject(handle, what)


def dare_layer_last_selection(handle, idx_ptr, count_ptr, batch_off_ptr, scores_ptr, delta_ptr, stream=0) -> int:
    return _lib.dare_layer_last_selection(handle, idx_ptr, count_ptr, batch_off_ptr, scores_ptr, delta_ptr, stream)


def dare_layer_read_caches(handle, k_ptr, v_ptr, o_ptr, q_prev_ptr, stream=0) -> int:
    return _lib.dare_layer_read_caches(handle, k_ptr, v_ptr, o_ptr, q_prev_ptr, stream)


def dare_layer_state_bytes(handle) -> int:
    return _lib.dare_layer_state_bytes(handle)


def dare_layer_export_state(handle, dst_ptr, nbytes, stream=0) -> int:
    return _lib.dare_layer_export_state(handle, dst_ptr, nbytes, stream)


def dare_layer_import_state(handle, src_ptr, nbytes, stream=0) -> int:
    return _lib.dare_layer_import_state(handle, src_ptr, nbytes, stream)


def dare_layer_last_launch_count(handle) -> int:
    return _lib.dare_layer_last_launch_count(handle)


def dare_layer_last_forms(handle) -> int:
    """FORM_* flags of the last step."""
    return _lib.dare_layer_last_forms(handle)


def dare_layer_set_profiling(handle, enable: int) -> int:
    return _lib.dare_layer_set_profiling(handle, enable)


def dare_layer_last_kernel_times(handle, slot_ptr, ms_ptr, capacity):
    """-> (status, n)"""
    n = C.c_int(0)
    st = _lib.dare_layer_last_kernel_times(handle, slot_ptr, ms_ptr, capacity, C.byref(n))
    return st, n.value


def dare_layer_debug_timestamps(handle, enable, out_ptr, stream=0) -> int:
    return _lib.dare_layer_debug_timestamps(handle, enable, out_ptr, stream)


def dare_drift_scores(q_now_ptr, q_prev_ptr, rows, head_dim, scores_ptr, stream=0) -> int:
    return _lib.dare_drift_scores(q_now_ptr, q_prev_ptr, rows, head_dim, scores_ptr, stream)


def dare_select_compact_scratch_bytes(n_tokens: int) -> int:
    return _lib.dare_select_compact_scratch_bytes(n_tokens)


def dare_select_compact(scores_ptr, n_tokens, threshold, idx_ptr, count_ptr, scratch_ptr, scratch_bytes, stream=0) -> int:
    return _lib.dare_select_compact(scores_ptr, n_tokens, threshold, idx_ptr, count_ptr, scratch_ptr, scratch_bytes,
                                    stream)


def dare_select_compact_static_max_tokens() -> int:
    return _lib.dare_select_compact_static_max_tokens()


def dare_select_compact_static(scores_ptr, n_tokens, threshold, idx_ptr, count_ptr, stream=0) -> int:
    """dare_select_compact without a scratch argument: for callers that may not allocate device memory."""
    return _lib.dare_select_compact_static(scores_ptr, n_tokens, threshold, idx_ptr, count_ptr, stream)


def dare_rope_table(cfg: RopeConfig, table_ptr, positions, stream=0) -> int:
    return _lib.dare_rope_table(C.byref(cfg) if cfg is not None else None, table_ptr, positions, stream)


def dare_rope(cfg: RopeApply, x_ptr, positions_ptr, table_ptr, y_ptr, status_ptr=None, stream=0) -> int:
    return _lib.dare_rope(C.byref(cfg) if cfg is not None else None, x_ptr, positions_ptr, table_ptr, y_ptr, status_ptr, stream)


def dare_linear(cfg: LinearConfig, x_ptr, w_ptr, bias_ptr, resid_ptr, y_ptr, status_ptr=None, stream=0) -> int:
    return _lib.dare_linear(C.byref(cfg) if cfg is not None else None, x_ptr, w_ptr, bias_ptr, resid_ptr, y_ptr, status_ptr,
                            stream)


def dare_attention_workspace_bytes(cfg: AttentionConfig) -> int:
    return _lib.dare_attention_workspace_bytes(C.byref(cfg) if cfg is not None else None)


def dare_attention(cfg: AttentionConfig, q_ptr, k_ptr, v_ptr, q_begin_ptr, k_begin_ptr, k_len_ptr, out_ptr, lse_ptr, workspace_ptr,
                   workspace_bytes, status_ptr=None, stream=0) -> int:
    return _lib.dare_attention(C.byref(cfg) if cfg is not None else None, q_ptr, k_ptr, v_ptr, q_begin_ptr, k_begin_ptr,
                               k_len_ptr, out_ptr, lse_ptr, workspace_ptr, workspace_bytes, status_ptr, stream)


def dare_kernel_slot_name(slot: int) -> str:
    return _lib.dare_kernel_slot_name(slot).decode()


def dare_stack_workspace_bytes(cfg: StackConfig) -> int:
    return _lib.dare_stack_workspace_bytes(C.byref(cfg))


def dare_stack_create(cfg: StackConfig, weights: StackWeights, workspace_ptr: int, workspace_bytes: int):
    """-> (status, handle)"""
    out = C.c_void_p()
    st = _lib.dare_stack_create(C.byref(cfg), C.byref(weights), workspace_ptr, workspace_bytes, C.byref(out))
    return st, out.value


def dare_stack_reset(handle) -> int:
    return _lib.dare_stack_reset(handle)


def dare_stack_destroy(handle) -> int:
    return _lib.dare_stack_destroy(handle)


def dare_stack_layer(handle, index: int):
    return _lib.dare_stack_layer(handle, index)


def dare_stack_forward(handle, tokens_ptr, batch, seq_total, seq_act, pos_begin, mode, taus_host_ptr, hidden_ptr,
                       stream=0) -> int:
    return _lib.dare_stack_forward(handle, tokens_ptr, batch, seq_total, seq_act, pos_begin, mode, taus_host_ptr,
                                   hidden_ptr, stream)


def dare_stack_set_capture(handle, layer_index, x_ptr, h_ptr) -> int:
    return _lib.dare_stack_set_capture(handle, layer_index, x_ptr, h_ptr)


def dare_stack_last_hidden(handle, dst_host_ptr, nbytes, stream=0) -> int:
    return _lib.dare_stack_last_hidden(handle, dst_host_ptr, nbytes, stream)


def dare_stack_decode_step(handle, tokens_ptr, batch, seq_total, prompt_len, block_index, first, mode, taus_host_ptr,
                           forced_pos_host_ptr, forced_tok_host_ptr, pos_out_ptr, tok_out_ptr, prob_out_ptr,
                           stream=0) -> int:
    return _lib.dare_stack_decode_step(handle, tokens_ptr, batch, seq_total, prompt_len, block_index, first, mode,
                                       taus_host_ptr, forced_pos_host_ptr, forced_tok_host_ptr, pos_out_ptr,
                                       tok_out_ptr, prob_out_ptr, stream)


# ---------------------------------------------------------------------------------------------------------------
def _current_stream(torch, device) -> int:
    """The current stream's handle without the Stream object around it (2.2 us a call, as long as a kernel launch)."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return raw(device.index)


# Stand-alone operators on torch tensors: argument marshalling, outputs and workspaces from torch's allocator, the tensors' device
# and its current stream.  `status`: an int32 CUDA tensor of one element that device-side problems are recorded in, or None.
# A call takes the host as long as several of the kernels behind it, so the wrappers ask each tensor for its shape and strides
# once, pack the argument block with struct and leave the wording of refusals to the ends that need one.
_torch = None


def _use_torch():
    global _torch, _DTYPES, _stream_of, _device_now
    import torch
    _DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
    _device_now = torch.cuda.current_device
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _stream_of = raw if raw is not None else (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch
    return torch


def _same_device(index, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != index:
            return False
    return index >= 0


def _status_ptr(status):
    if status is None:
        return None
    if status.dtype != _torch.int32 or status.numel() < 1:
        raise ValueError("status: int32 tensor of one element expected")
    return status.data_ptr()


def _call(fn, name, index, *args):
    """fn(*args, stream) with the tensors' device current."""
    if _device_now() == index:
        st = fn(*args, _stream_of(index))
    else:
        with _torch.cuda.device(index):
            st = fn(*args, _stream_of(index))
    if st != OK:
        raise DareError(st, name)


def rope_table(positions, rotary_dim, theta, scaling=ROPE_SCALE["none"], factor=1.0, trained=0, low=1.0, high=32.0,
               magnitude=1.0, device="cuda", out=None):
    """-> float32 [positions, rotary_dim / 2, 2]: cosines and sines of dare_rope_table, for `rope`."""
    torch = _torch or _use_torch()
    shape = (positions, rotary_dim // 2, 2)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=device)
    index = out.get_device()
    if index < 0 or out.dtype != torch.float32 or out.shape != shape or not out.is_contiguous():
        raise ValueError("out: contiguous float32 CUDA tensor [positions, rotary_dim / 2, 2] expected")
    cfg = RopeConfig(C.sizeof(RopeConfig), rotary_dim, theta, scaling, trained, factor, low, high, magnitude)
    _call(_lib.dare_rope_table, "dare_rope_table", index, C.byref(cfg), out.data_ptr(), positions)
    return out


_ROPE_APPLY = struct.Struct("=Iiqiiiiii5q")           # RopeApply


def rope(x, table, positions=None, layout=ROPE_LAYOUT["half"], transpose=False, pos_begin=0, out=None, status=None):
    """x [tokens, heads, head_dim] (any token and head strides) with its heads turned by the table's rows of `positions` (int32
    [tokens]; None: pos_begin, pos_begin + 1, ...).  The table's width gives the part of the head that turns.  out may be x."""
    torch = _torch or _use_torch()
    dt, index = _DTYPES.get(x.dtype), x.get_device()
    if dt is None or x.dim() != 3 or table.dtype != torch.float32 or table.dim() != 3 or not _same_device(index, table, positions, out, status):
        raise ValueError("x: bf16 or float32 CUDA tensor [tokens, heads, head_dim], table: float32 [positions, rotary_dim / 2, 2] on its "
                         "device expected")
    tokens, heads, hd = shape = x.shape
    xt, xh, xe = x.stride()
    rows, pairs, two = table.shape
    if out is None:
        out = torch.empty(tokens, heads, hd, dtype=x.dtype, device=x.device)
        yt, yh, ye = heads * hd, hd, 1
    else:
        yt, yh, ye = out.stride()
        if out.shape != shape or out.dtype != x.dtype:
            raise ValueError("out: as x")
    if hd > 1 and (xe != 1 or ye != 1):
        raise ValueError("the elements of a head have to lie side by side")
    if two != 2 or not table.is_contiguous():
        raise ValueError("table: contiguous [positions, rotary_dim / 2, 2] expected")
    pos = None
    if positions is not None:
        if positions.dtype != torch.int32 or positions.shape != shape[:1] or not positions.is_contiguous():
            raise ValueError("positions: contiguous int32 [tokens] expected")
        pos = positions.data_ptr()
    cfg = _ROPE_APPLY.pack(_ROPE_APPLY.size, dt, tokens, heads, hd, 2 * pairs, layout, 1 if transpose else 0, pos_begin, xt, xh, yt,
                           yh, rows)
    _call(_fast_rope, "dare_rope", index, cfg, x.data_ptr(), pos, table.data_ptr(), out.data_ptr(),
          _status_ptr(status))
    return out


_LINEAR = struct.Struct("=Iiqiiii4q")                 # LinearConfig


def linear(x, w, bias=None, act=ACT["none"], resid=None, out=None, status=None):
    """act(x w^T + bias) + resid: x [..., in_features], w [out_features, in_features] (as the layer's weights), bias float32
    [out_features], resid [..., out_features].  Rows may be strided; out may be resid."""
    torch = _torch or _use_torch()
    dtype, index = x.dtype, x.get_device()
    dt = _DTYPES.get(dtype)
    if dt is None or w.dtype != dtype or w.dim() != 2 or not _same_device(index, w, bias, resid, out, status):
        raise ValueError("x: bf16 or float32 CUDA tensor, w: [out_features, in_features] of its type and device expected")
    n, k = w.shape
    shape = x.shape
    if shape[-1] != k:
        raise ValueError("x and w: in_features differ")
    flat = len(shape) == 2
    x2 = x if flat else x.reshape(-1, k)
    m = x2.shape[0]
    shape = (m, n) if flat else shape[:-1] + (n,)
    if out is None:
        out = torch.empty(*shape, dtype=dtype, device=x.device)           # (sizes one by one: a tuple of them costs a microsecond)
    elif out.shape != shape or out.dtype != dtype:
        raise ValueError("out: [..., out_features] of x's type expected")
    y2 = out if flat else out.view(-1, n)
    r2, rr, re = resid, 0, 1
    if resid is not None:
        if resid.shape != shape or resid.dtype != dtype:
            raise ValueError("resid: [..., out_features] of x's type expected")
        r2 = resid if flat else resid.view(-1, n)
        rr, re = r2.stride()
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (n,) or not bias.is_contiguous()):
        raise ValueError("bias: contiguous float32 [out_features] expected")
    (xr, xe), (wr, we), (yr, ye) = x2.stride(), w.stride(), y2.stride()
    if (k > 1 and (xe != 1 or we != 1)) or (n > 1 and (ye != 1 or re != 1)):
        raise ValueError("the elements of a row have to lie side by side")
    cfg = _LINEAR.pack(_LINEAR.size, dt, m, k, n, act, 0, xr, wr, rr, yr)
    _call(_fast_linear, "dare_linear", index, cfg, x2.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(),
          None if r2 is None else r2.data_ptr(), y2.data_ptr(), _status_ptr(status))
    return out


_ATTENTION = struct.Struct("=Iiiiiiif10q")            # AttentionConfig


def attention(q, k, v, q_begin, k_begin, k_len=None, causal=False, scale=None, out=None, return_lse=False, status=None):
    """Softmax attention over packed sequences: q [q_rows, n_heads, head_dim], k and v [k_rows, n_kv_heads, head_dim] (any row and
    head strides); q_begin int32 [batch + 1], k_begin int32 [batch + 1] or, with k_len int32 [batch], [batch].  scale: None for
    head_dim^-0.5.  -> out, or (out, lse float32 [q_rows, n_heads])."""
    torch = _torch or _use_torch()
    dtype, index = q.dtype, q.get_device()
    dt = _DTYPES.get(dtype)
    if dt is None or k.dtype != dtype or v.dtype != dtype or not _same_device(index, k, v, q_begin, k_begin, k_len, out, status):
        raise ValueError("q, k, v: bf16 or float32 CUDA tensors of one type, everything on one device expected")
    shape = q.shape
    rows, heads, hd = shape
    k_rows, kv_heads, k_hd = k.shape
    if k_hd != hd or v.shape != k.shape:
        raise ValueError("q: [rows, heads, head_dim], k and v: [rows, kv heads, head_dim] expected")
    batch = q_begin.shape[0] - 1
    i32 = torch.int32
    if (q_begin.dtype != i32 or k_begin.dtype != i32 or q_begin.dim() != 1 or k_begin.dim() != 1 or not q_begin.is_contiguous() or
            not k_begin.is_contiguous() or k_begin.shape[0] < (batch + 1 if k_len is None else batch) or
            (k_len is not None and (k_len.dtype != i32 or k_len.dim() != 1 or k_len.shape[0] < batch or not k_len.is_contiguous()))):
        raise ValueError("q_begin, k_begin, k_len: contiguous int32 [batch + 1], [batch + 1] (with k_len: [batch]), [batch] expected")
    qt, qh, qe = q.stride()
    kt, kh, ke = k.stride()
    vt, vh, ve = v.stride()
    if out is None:
        out = torch.empty(rows, heads, hd, dtype=dtype, device=q.device)
        ot, oh, oe = heads * hd, hd, 1
    else:
        ot, oh, oe = out.stride()
        if out.shape != shape or out.dtype != dtype:
            raise ValueError("out: as q")
    if qe != 1 or ke != 1 or ve != 1 or oe != 1:
        raise ValueError("the elements of a head have to lie side by side")
    cfg = _ATTENTION.pack(_ATTENTION.size, dt, batch, heads, kv_heads, hd, 1 if causal else 0, hd ** -0.5 if scale is None else scale, rows,
                          k_rows, qt, qh, kt, kh, vt, vh, ot, oh)
    nbytes = _fast_attention_bytes(cfg)
    work = torch.empty(nbytes or 16, dtype=torch.uint8, device=q.device)
    lse = torch.empty(rows, heads, dtype=torch.float32, device=q.device) if return_lse else None
    _call(_fast_attention, "dare_attention", index, cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), q_begin.data_ptr(),
          k_begin.data_ptr(), None if k_len is None else k_len.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(),
          work.data_ptr(), nbytes, _status_ptr(status))
    return (out, lse) if return_lse else out


def _packed_entry(name, rest, res=C.c_int):
    """The entry point with its argument block given as bytes."""
    return C.CFUNCTYPE(res, C.c_char_p, *rest)((name, _lib))


_fast_rope = _packed_entry("dare_rope", [C.c_void_p] * 6)
_fast_linear = _packed_entry("dare_linear", [C.c_void_p] * 7)
_fast_attention = _packed_entry("dare_attention", [C.c_void_p] * 9 + [C.c_size_t] + [C.c_void_p] * 2)
_fast_attention_bytes = _packed_entry("dare_attention_workspace_bytes", [], C.c_size_t)


class Layer:
    """Convenience wrapper: owns the torch tensors behind a handle (weights, workspace) and marshals pointers.

    No arithmetic happens here.  `x`/`y` are torch CUDA tensors (or pinned host tensors for `step_host`).
    """

    def __init__(self, shape, weights: dict, device="cuda:0", kernel_path=PATH_AUTO, max_batch=None, max_seq=None,
                 score_head=0):
        import numpy as np
        import torch
        self.torch = torch
        self.shape = shape
        self.device = torch.device(device)
        self.tdtype = torch.bfloat16 if shape.dtype == BF16 else torch.float32
        self.max_batch = max_batch or shape.batch
        self.max_seq = max_seq or shape.seq
        self.cfg = make_config(shape.d_model, shape.n_heads, shape.head_dim, self.max_batch, self.max_seq,
                               shape.rope_theta, shape.rms_eps, shape.dtype, score_head, kernel_path)
        self._w = {}
        for k in ("w_q", "w_k", "w_v", "w_o"):
            v = weights[k]
            t = v if isinstance(v, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(v, np.float32))
            self._w[k] = t.to(self.device, self.tdtype).contiguous()
        g = weights["rms_gain"]
        g = g if isinstance(g, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(g, np.float32))
        self._w["rms_gain"] = g.to(self.device, torch.float32).contiguous()
        self.wstruct = LayerWeights(*(self._w[k].data_ptr() for k in ("w_q", "w_k", "w_v", "w_o", "rms_gain")))
        nbytes = dare_layer_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise DareError(ERR_UNSUPPORTED, "dare_layer_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        with torch.cuda.device(self.device):
            st, self.handle = dare_layer_create(self.cfg, self.wstruct, base, nbytes)
        if st != OK:
            raise DareError(st, "dare_layer_create")

    def _stream(self):
        return _current_stream(self.torch, self.device)

    def step(self, x, mode, threshold, y=None, pos_begin=0):
        torch = self.torch
        assert x.is_cuda and x.dtype == self.tdtype and x.is_contiguous()
        if y is None:
            y = torch.empty_like(x)
        st = dare_layer_step(self.handle, x.data_ptr(), x.shape[0], x.shape[1], pos_begin, mode, threshold,
                             y.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_step")
        return y

    def step_quantile(self, x, mode, reuse_count, y=None, pos_begin=0):
        """The step with the threshold taken from its own scores: the `reuse_count` least-drifted tokens are reused."""
        torch = self.torch
        assert x.is_cuda and x.dtype == self.tdtype and x.is_contiguous()
        if y is None:
            y = torch.empty_like(x)
        st = dare_layer_step_quantile(self.handle, x.data_ptr(), x.shape[0], x.shape[1], pos_begin, mode, reuse_count,
                                      y.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_step_quantile")
        return y

    def last_threshold(self) -> float:
        st, tau = dare_layer_last_threshold(self.handle, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_last_threshold")
        return tau

    def step_host(self, x_host, mode, threshold, y_host, pos_begin=0):
        st = dare_layer_step_host(self.handle, x_host.data_ptr(), x_host.shape[0], x_host.shape[1], pos_begin, mode,
                                  threshold, y_host.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_step_host")
        return y_host

    def step_host_async(self, x_host, mode, threshold, y_host, pos_begin=0):
        """Enqueue only: y_host is defined after wait_host(); x_host must stay valid until then."""
        st = dare_layer_step_host_async(self.handle, x_host.data_ptr(), x_host.shape[0], x_host.shape[1], pos_begin, mode,
                                        threshold, y_host.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_step_host_async")

    def wait_host(self):
        st = dare_layer_wait_host(self.handle)
        if st != OK:
            raise DareError(st, "dare_layer_wait_host")

    def reset(self):
        st = dare_layer_reset(self.handle)
        if st != OK:
            raise DareError(st, "dare_layer_reset")

    def status(self) -> int:
        return dare_layer_status(self.handle, self._stream())

    def clear_status(self):
        st = dare_layer_clear_status(self.handle, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_clear_status")

    def wait_probe(self, limit_ns):
        st, waited = dare_layer_debug_wait_probe(self.handle, limit_ns, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_debug_wait_probe")
        return waited

    def inject(self, what):
        st = dare_layer_debug_inject(self.handle, what)
        if st != OK:
            raise DareError(st, "dare_layer_debug_inject")

    def last_selection(self, batch, seq_act):
        """-> dict(idx, count, batch_off, scores, delta) as numpy arrays."""
        import numpy as np
        T = batch * seq_act
        idx = np.zeros(T, np.int32)
        cnt = np.zeros(1, np.int32)
        boff = np.zeros(batch + 1, np.int32)
        sc = np.zeros(T, np.float32)
        dl = np.zeros(T, np.int32)
        st = dare_layer_last_selection(self.handle, idx.ctypes.data, cnt.ctypes.data, boff.ctypes.data,
                                       sc.ctypes.data, dl.ctypes.data, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_last_selection")
        n = int(cnt[0])
        return {"idx": idx[:n].copy(), "count": n, "batch_off": boff, "scores": sc, "delta": dl.reshape(batch, seq_act)}

    def read_caches(self, batch, kv_len):
        """-> dict(k, v, o, q_prev) as float32 numpy arrays [batch, kv_len, ...]."""
        import numpy as np
        torch = self.torch
        d, hd = self.shape.d_model, self.shape.head_dim
        host = [torch.empty((batch, kv_len, d), dtype=self.tdtype) for _ in range(3)]
        qp = np.zeros((batch, kv_len, hd), np.float32)
        st = dare_layer_read_caches(self.handle, host[0].data_ptr(), host[1].data_ptr(), host[2].data_ptr(),
                                    qp.ctypes.data, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_read_caches")
        k, v, o = (h.float().numpy() for h in host)
        return {"k": k, "v": v, "o": o, "q_prev": qp}

    def set_profiling(self, enable: bool):
        st = dare_layer_set_profiling(self.handle, 1 if enable else 0)
        if st != OK:
            raise DareError(st, "dare_layer_set_profiling")

    def kernel_times(self):
        """-> list of (kernel name, milliseconds) of the last step, in launch order (profiling must be on)."""
        import numpy as np
        slots = np.zeros(16, np.int32)
        ms = np.zeros(16, np.float32)
        st, n = dare_layer_last_kernel_times(self.handle, slots.ctypes.data, ms.ctypes.data, 16)
        if st != OK:
            raise DareError(st, "dare_layer_last_kernel_times")
        return [(dare_kernel_slot_name(int(slots[i])), float(ms[i])) for i in range(n)]

    def debug_timestamps(self, enable=True):
        """-> uint64[8, 8] phase timestamps (ns) of the tensor-core kernels of the last step; see include/dare.h."""
        import numpy as np
        out = np.zeros(64 + 3 * 1024, np.uint64)
        st = dare_layer_debug_timestamps(self.handle, 1 if enable else 0, out.ctypes.data, self._stream())
        if st != OK:
            raise DareError(st, "dare_layer_debug_timestamps")
        self.debug_blocks = out[64:].reshape(1024, 3)
        return out[:64].reshape(8, 8)

    def launch_count(self) -> int:
        return dare_layer_last_launch_count(self.handle)

    def forms(self) -> int:
        return dare_layer_last_forms(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            dare_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _LayerView(Layer):
    """A layer that belongs to a stack: same observation calls, no ownership."""

    def __init__(self, handle, shape, torch, device):
        self.handle, self.shape, self.torch, self.device = handle, shape, torch, device
        self.tdtype = torch.bfloat16

    def close(self):
        self.handle = None


class Stack:
    """Convenience wrapper around dare_stack_*: owns the device copies of the weights and the workspace."""

    def __init__(self, sshape, weights: dict, batch: int, device="cuda:0"):
        import numpy as np
        import torch
        self.torch, self.sshape, self.batch = torch, sshape, batch
        self.device = torch.device(device)
        lay = sshape.layer
        dev = lambda a, dt: (a if isinstance(a, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(a, np.float32))) \
            .to(self.device, dt).contiguous()
        bf, f32 = torch.bfloat16, torch.float32
        self._keep = [dev(weights["emb"], bf), dev(weights["head"], bf), dev(weights["final_gain"], f32)]
        blocks = (BlockWeights * sshape.n_layers)()
        for l, lw in enumerate(weights["layers"]):
            t = {k: dev(lw[k], bf) for k in ("w_q", "w_k", "w_v", "w_o", "w_gate", "w_up", "w_down")}
            t["rms_gain"], t["gain2"] = dev(lw["rms_gain"], f32), dev(lw["gain2"], f32)
            self._keep.append(t)
            blocks[l] = BlockWeights(LayerWeights(t["w_q"].data_ptr(), t["w_k"].data_ptr(), t["w_v"].data_ptr(),
                                                  t["w_o"].data_ptr(), t["rms_gain"].data_ptr()),
                                     t["gain2"].data_ptr(), t["w_gate"].data_ptr(), t["w_up"].data_ptr(),
                                     t["w_down"].data_ptr())
        self._blocks = blocks
        lcfg = make_config(lay.d_model, lay.n_heads, lay.head_dim, batch, lay.seq, lay.rope_theta, lay.rms_eps, BF16, 0,
                           PATH_TENSOR)
        self.cfg = StackConfig(C.sizeof(StackConfig), sshape.n_layers, sshape.d_ff, sshape.vocab, sshape.mask_id,
                               lay.block, lcfg)
        self.w = StackWeights(self._keep[0].data_ptr(), self._keep[1].data_ptr(), self._keep[2].data_ptr(), blocks)
        nbytes = dare_stack_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise DareError(ERR_UNSUPPORTED, "dare_stack_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        with torch.cuda.device(self.device):
            st, self.handle = dare_stack_create(self.cfg, self.w, base, nbytes)
        if st != OK:
            raise DareError(st, "dare_stack_create")

    def _stream(self):
        return _current_stream(self.torch, self.device)

    def layer(self, index: int) -> "_LayerView":
        return _LayerView(dare_stack_layer(self.handle, index), self.sshape.layer, self.torch, self.device)

    def reset(self):
        dare_stack_reset(self.handle)

    def forward(self, tokens, seq_act, pos_begin, mode, taus):
        """tokens: int32 CUDA tensor [batch, seq_total]; -> bf16 hidden states [batch, seq_act, d_model]."""
        import numpy as np
        torch = self.torch
        taus = np.ascontiguousarray(taus, np.float32)
        out = torch.empty((tokens.shape[0], seq_act, self.sshape.layer.d_model), dtype=torch.bfloat16, device=self.device)
        st = dare_stack_forward(self.handle, tokens.data_ptr(), tokens.shape[0], tokens.shape[1], seq_act, pos_begin, mode,
                                taus.ctypes.data, out.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_stack_forward")
        return out

    def decode_step(self, tokens, prompt_len, block_index, first, mode, taus, forced=None):
        """-> (pos, tok, prob) numpy arrays [batch]: the step's own choice; `tokens` is updated in place."""
        import numpy as np
        torch = self.torch
        B = tokens.shape[0]
        taus = np.ascontiguousarray(taus, np.float32)
        pos = torch.empty(B, dtype=torch.int32, device=self.device)
        tok = torch.empty(B, dtype=torch.int32, device=self.device)
        prob = torch.empty(B, dtype=torch.float32, device=self.device)
        fp = ft = None
        if forced is not None:
            fp = np.ascontiguousarray(forced[0], np.int32)
            ft = np.ascontiguousarray(forced[1], np.int32)
        st = dare_stack_decode_step(self.handle, tokens.data_ptr(), B, tokens.shape[1], prompt_len, block_index,
                                    1 if first else 0, mode, taus.ctypes.data,
                                    fp.ctypes.data if fp is not None else None, ft.ctypes.data if ft is not None else None,
                                    pos.data_ptr(), tok.data_ptr(), prob.data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_stack_decode_step")
        torch.cuda.synchronize(self.device)       # the forced arrays are host memory read by an async copy
        return pos.cpu().numpy(), tok.cpu().numpy(), prob.cpu().numpy()

    def decode_step_enqueue(self, tokens, prompt_len, block_index, first, mode, taus, out=None):
        """Enqueue-only form of decode_step (no forced choice, no synchronisation, nothing allocated when `out` is
        given): usable inside a CUDA-graph capture.  -> (pos, tok, prob) device tensors [batch]."""
        import numpy as np
        torch = self.torch
        B = tokens.shape[0]
        taus = np.ascontiguousarray(taus, np.float32)
        if out is None:
            out = (torch.empty(B, dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.float32, device=self.device))
        st = dare_stack_decode_step(self.handle, tokens.data_ptr(), B, tokens.shape[1], prompt_len, block_index,
                                    1 if first else 0, mode, taus.ctypes.data, None, None,
                                    out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), self._stream())
        if st != OK:
            raise DareError(st, "dare_stack_decode_step")
        return out

    def set_capture(self, layer_index, x_buf=None, h_buf=None):
        st = dare_stack_set_capture(self.handle, layer_index, x_buf.data_ptr() if x_buf is not None else None,
                                    h_buf.data_ptr() if h_buf is not None else None)
        if st != OK:
            raise DareError(st, "dare_stack_set_capture")

    def last_hidden(self, batch, seq_act):
        """-> float32 numpy [batch, seq_act, d_model]: final-normed states of the last pass."""
        torch = self.torch
        h = torch.empty((batch, seq_act, self.sshape.layer.d_model), dtype=torch.bfloat16)
        st = dare_stack_last_hidden(self.handle, h.data_ptr(), h.numel() * 2, self._stream())
        if st != OK:
            raise DareError(st, "dare_stack_last_hidden")
        return h.float().numpy()

    def close(self):
        if getattr(self, "handle", None):
            dare_stack_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
