"""ctypes binding with the same names as include/csbrnn.h and include/csbrnn_lm.h (argument marshalling only).

`stream` (None: the current stream) is the stream that a call runs on.  Another one has to be made to wait for what produced the arguments,
and they have to live until it is done; workspaces and new results are safe on it, and results may be dropped while the
caller's stream still reads them.

Nothing here has a gradient.  The language-model operators (delta_*, adapter_add, verify_drafts, short_conv, selective_scan, block_norm, sample) refuse operands that require one while
gradients are enabled, and operands that are not on the current device.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import sys
from typing import List, Optional, Sequence

import numpy as np

CELL_LSTM = 0
CELL_GRU = 1
CELL_LSTMP = 2
CELL_LIGRU = 3
CELL_GRU_RB = 4
VAL_F32, VAL_F16, VAL_BF16 = 0, 1, 2

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libcsbrnn.so")
_lib = None
_raw_delta = {}
_raw = {}

# every symbol the headers under include/ declare
SYMBOLS = ["csb_last_error", "csb_pack", "csb_view_get", "csb_unpack", "csb_set_value_format", "csb_value_format", "csb_sharing_model", "csb_plan", "csb_plan_ex", "csb_plan_rows", "csb_plan_stats_get", "csb_plan_validate", "csb_status",
           "csb_device_bytes", "csb_upload", "csb_workspace_bytes", "csb_spmv", "csb_spmv_static_limit", "csb_spmv_static", "csb_spmm", "csb_spmm_bfloat", "csb_spmm_half",
           "csb_debug_stamp_count", "csb_debug_spmv_stamps",
           "csb_debug_stream_read_out_floats", "csb_debug_stream_read", "csb_debug_spmm_columns", "csb_debug_quad_passes", "csb_debug_spmm_force", "csb_debug_spmm_form", "csb_debug_spmm_panel", "csb_debug_rnn_prefers_resident",
           "csb_project_workspace_bytes", "csb_project", "csb_rnn_create_lstmp", "csb_rnn_create_gru_rb",
           "csb_rnn_create", "csb_rnn_device_bytes", "csb_rnn_upload", "csb_rnn_plan_resident", "csb_rnn_stats",
           "csb_rnn_set_poll_limit", "csb_rnn_status", "csb_rnn_workspace_bytes", "csb_rnn_forward", "csb_free", "csb_rnn_free",
           # include/csbrnn_lm.h
           "csb_delta_recurrent", "csb_delta_workspace_bytes", "csb_delta_chunked", "csb_adapter_workspace_bytes", "csb_adapter_add",
           "csb_verify_workspace_bytes", "csb_verify_drafts", "csb_short_conv", "csb_scan_workspace_bytes", "csb_selective_scan",
           "csb_block_norm", "csb_sample_workspace_bytes", "csb_sample"]


class csb_sharing_stats(C.Structure):
    _fields_ = [("work", C.c_int64), ("iterations", C.c_int64), ("cycles_none", C.c_int64),
                ("cycles_horizontal", C.c_int64), ("cycles_vertical", C.c_int64), ("cycles_2d", C.c_int64),
                ("eff_none", C.c_double), ("eff_horizontal", C.c_double), ("eff_vertical", C.c_double),
                ("eff_2d", C.c_double), ("exact_2d", C.c_int32), ("reserved", C.c_int32)]


class CsbError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"csb error {code}: {msg}")
        self.code = code


class csb_view(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64),
                ("br", C.c_int32), ("bc", C.c_int32), ("nbr", C.c_int32), ("nbc", C.c_int32),
                ("nnz", C.c_int64), ("n_rowidx", C.c_int64), ("n_colidx", C.c_int64),
                ("nrows", C.POINTER(C.c_int32)), ("ncols", C.POINTER(C.c_int32)),
                ("rowidx", C.POINTER(C.c_uint16)), ("colidx", C.POINTER(C.c_uint16)),
                ("val", C.POINTER(C.c_float)),
                ("val_off", C.POINTER(C.c_int64)), ("row_off", C.POINTER(C.c_int64)),
                ("col_off", C.POINTER(C.c_int64))]


class csb_rnn_plan_stats(C.Structure):
    _fields_ = [("resident", C.c_int32), ("n_workgroups", C.c_int32), ("slots_per_lane", C.c_int32),
                ("reserved", C.c_int32), ("slot_fill", C.c_double), ("lanes_max_over_mean", C.c_double)]


class csb_plan_stats(C.Structure):
    _fields_ = [("n_chunks", C.c_int32), ("waves_per_chunk", C.c_int32), ("n_groups", C.c_int32),
                ("n_shared_tiles", C.c_int32), ("work_max", C.c_double), ("work_mean", C.c_double),
                ("lane_fill", C.c_double), ("nosplit_max_over_mean", C.c_double),
                ("chunk_max_over_mean", C.c_double), ("whole_tiles", C.c_int32), ("row_owned", C.c_int32),
                ("rounds", C.c_int32), ("reserved", C.c_int32), ("matvec_bytes", C.c_int64)]


class csb_delta_args(C.Structure):
    _fields_ = [("type", C.c_int32), ("heads_k", C.c_int32), ("heads_v", C.c_int32), ("dk", C.c_int32), ("dv", C.c_int32),
                ("n_seq", C.c_int32), ("n_tokens", C.c_int64), ("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("ldq", C.c_int64), ("ldk", C.c_int64), ("ldv", C.c_int64), ("d_g", C.c_void_p), ("d_beta", C.c_void_p),
                ("ldg", C.c_int64), ("ldbeta", C.c_int64), ("d_start", C.c_void_p), ("d_len", C.c_void_p),
                ("d_state_in", C.c_void_p), ("d_state_out", C.c_void_p), ("d_slot", C.c_void_p), ("n_states", C.c_int32),
                ("scale", C.c_float), ("d_out", C.c_void_p), ("ldo", C.c_int64)]


class csb_conv_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("type", "channels", "width", "silu", "n_seq", "n_states")] + [
        ("n_tokens", C.c_int64), ("d_x", C.c_void_p), ("ldx", C.c_int64)] + [
        (n, C.c_void_p) for n in ("d_w", "d_bias", "d_start", "d_len", "d_state_in", "d_state_out", "d_slot", "d_out")] + [("ldo", C.c_int64)]


class csb_scan_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("type", "channels", "groups", "n", "softplus", "n_seq")] + [("n_tokens", C.c_int64)] + [
        (n, C.c_void_p) for n in ("d_x", "d_dt", "d_z", "d_B", "d_C")] + [(n, C.c_int64) for n in ("ldx", "lddt", "ldz", "ldB", "ldC")] + [
        (n, C.c_void_p) for n in ("d_A", "d_D", "d_dt_bias", "d_start", "d_len", "d_state_in", "d_state_out", "d_slot")] + [
        ("n_states", C.c_int32), ("reserved", C.c_int32), ("d_out", C.c_void_p), ("ldo", C.c_int64)]


class csb_norm_operand(C.Structure):
    _fields_ = [("d", C.c_void_p), ("ld", C.c_int64), ("type", C.c_int32), ("columns", C.c_int32)]


class csb_norm_args(C.Structure):
    _fields_ = [("n_tokens", C.c_int64)] + [(n, C.c_int32) for n in ("width", "groups", "after", "before", "gate_kind", "gate_first")] + [
        ("scale", C.c_float), ("eps", C.c_float)] + [(n, csb_norm_operand) for n in ("y", "gate", "x", "r", "out")] + [
        (n, C.c_void_p) for n in ("d_after_w", "d_after_b", "d_scale", "d_before_w", "d_before_b")]


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libcsbrnn.so; fails loudly if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2005_05758_amd.build` "
                          "(there is no CPU fallback)")
    L = C.CDLL(_LIB_PATH)
    L.csb_last_error.restype = C.c_char_p
    L.csb_pack.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]
    L.csb_view_get.argtypes = [C.c_void_p, C.POINTER(csb_view)]
    L.csb_unpack.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
    L.csb_sharing_model.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(csb_sharing_stats)]
    L.csb_set_value_format.argtypes = [C.c_void_p, C.c_int32]
    L.csb_value_format.argtypes = [C.c_void_p]
    L.csb_plan.argtypes = [C.c_void_p, C.c_int32, C.POINTER(csb_plan_stats)]
    L.csb_plan_ex.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(csb_plan_stats)]
    L.csb_plan_rows.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(csb_plan_stats)]
    L.csb_plan_stats_get.argtypes = [C.c_void_p, C.POINTER(csb_plan_stats)]
    L.csb_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
    L.csb_rnn_set_poll_limit.argtypes = [C.c_void_p, C.c_uint32]
    L.csb_rnn_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
    L.csb_plan_validate.argtypes = [C.c_void_p]
    L.csb_device_bytes.argtypes = [C.c_void_p]
    L.csb_device_bytes.restype = C.c_size_t
    L.csb_upload.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.csb_workspace_bytes.argtypes = [C.c_void_p, C.c_int32]
    L.csb_workspace_bytes.restype = C.c_size_t
    L.csb_spmv.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    L.csb_spmv_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    L.csb_spmv_static_limit.argtypes = []
    L.csb_spmv_static_limit.restype = C.c_size_t
    L.csb_debug_stamp_count.argtypes = [C.c_void_p]
    L.csb_debug_stamp_count.restype = C.c_size_t
    L.csb_debug_spmv_stamps.argtypes = [C.c_void_p] * 6
    L.csb_debug_stream_read_out_floats.argtypes = []
    L.csb_debug_stream_read_out_floats.restype = C.c_size_t
    L.csb_debug_stream_read.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    L.csb_debug_spmm_columns.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
    L.csb_debug_spmm_force.argtypes = [C.c_void_p, C.c_int32]
    L.csb_debug_spmm_form.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
    L.csb_debug_spmm_panel.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
    L.csb_debug_quad_passes.argtypes = [C.c_void_p, C.c_int32]
    L.csb_debug_quad_passes.restype = C.c_int64
    L.csb_debug_rnn_prefers_resident.argtypes = [C.c_void_p, C.c_int32]
    L.csb_project_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int32, C.c_int32]
    L.csb_project_workspace_bytes.restype = C.c_size_t
    L.csb_project.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_double,
                              C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
    L.csb_spmm.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
    L.csb_spmm_bfloat.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
    L.csb_spmm_half.argtypes = L.csb_spmm_bfloat.argtypes
    L.csb_rnn_create.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_void_p),
                                 C.POINTER(C.c_void_p), C.POINTER(C.c_void_p)]
    L.csb_rnn_create_lstmp.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_void_p),
                                       C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p)]
    L.csb_rnn_create_gru_rb.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_void_p),
                                        C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p)]
    L.csb_rnn_device_bytes.argtypes = [C.c_void_p]
    L.csb_rnn_device_bytes.restype = C.c_size_t
    L.csb_rnn_upload.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.csb_rnn_plan_resident.argtypes = [C.c_void_p, C.c_int32]
    L.csb_rnn_stats.argtypes = [C.c_void_p, C.POINTER(csb_rnn_plan_stats)]
    L.csb_rnn_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    L.csb_rnn_workspace_bytes.restype = C.c_size_t
    L.csb_rnn_forward.argtypes = [C.c_void_p] + [C.c_void_p] * 6 + [C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
    L.csb_delta_recurrent.argtypes = [C.POINTER(csb_delta_args), C.c_void_p]
    L.csb_delta_chunked.argtypes = [C.POINTER(csb_delta_args), C.c_void_p, C.c_void_p]
    L.csb_delta_workspace_bytes.argtypes = [C.POINTER(csb_delta_args)]
    L.csb_delta_workspace_bytes.restype = C.c_size_t
    L.csb_adapter_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32]
    L.csb_adapter_workspace_bytes.restype = C.c_size_t
    L.csb_adapter_add.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int32,
                                  C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p]
    L.csb_verify_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    L.csb_verify_workspace_bytes.restype = C.c_size_t
    L.csb_verify_drafts.argtypes = [C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64] + [C.c_void_p] * 4 + \
                                   [C.c_int32] * 3 + [C.c_void_p] * 4
    L.csb_short_conv.argtypes = [C.POINTER(csb_conv_args), C.c_void_p]
    L.csb_scan_workspace_bytes.argtypes = [C.POINTER(csb_scan_args)]
    L.csb_scan_workspace_bytes.restype = C.c_size_t
    L.csb_selective_scan.argtypes = [C.POINTER(csb_scan_args), C.c_void_p, C.c_void_p]
    L.csb_block_norm.argtypes = [C.POINTER(csb_norm_args), C.c_void_p]
    L.csb_sample_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    L.csb_sample_workspace_bytes.restype = C.c_size_t
    L.csb_sample.argtypes = [C.c_int32, C.c_void_p, C.c_int64] + [C.c_void_p] * 5 + [C.c_int32] * 2 + [C.c_void_p] * 2 + [C.c_int64] + [C.c_void_p] * 2
    L.csb_free.argtypes = [C.c_void_p]
    L.csb_free.restype = None
    L.csb_rnn_free.argtypes = [C.c_void_p]
    L.csb_rnn_free.restype = None
    for name in SYMBOLS:
        fn = getattr(L, name)
        if fn.restype is C.c_int and name not in ("csb_free", "csb_rnn_free"):
            fn.restype = C.c_int
    # the same entry points taking csb_delta_args as bytes: filling a ctypes structure of 26 fields takes 2 us, a small call's kernel is done in 5
    for key, name in (("recurrent", "csb_delta_recurrent"), ("chunked", "csb_delta_chunked"), ("workspace", "csb_delta_workspace_bytes")):
        fn = L[name]
        fn.argtypes = [C.c_char_p] + [C.c_void_p] * {"recurrent": 1, "chunked": 2, "workspace": 0}[key]
        fn.restype = C.c_size_t if key == "workspace" else C.c_int
        _raw_delta[key] = fn
    for name, more in (("csb_short_conv", 1), ("csb_scan_workspace_bytes", 0), ("csb_selective_scan", 2), ("csb_block_norm", 1)):      # (the same for these)
        fn = L[name]
        fn.argtypes = [C.c_char_p] + [C.c_void_p] * more
        fn.restype = C.c_int if more else C.c_size_t
        _raw[name] = fn
    _lib = L
    return L


def lib():
    return load_library()


def _check(rc: int):
    if rc != 0:
        raise CsbError(rc, lib().csb_last_error().decode())


def _f32():
    import torch
    return torch.float32


def _dptr(t, dtype=None) -> Optional[int]:
    """Device pointer of a contiguous torch tensor (or None); `dtype`: what the callee reads it as."""
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    if dtype is not None:
        assert t.dtype is dtype, f"expected a {dtype} tensor, got {t.dtype}"
    return t.data_ptr()


def _stream_ptr(stream=None) -> Optional[int]:
    """Handle of `stream`, or of the current stream of the current device (None: the default stream).
    Asked for as a number: building a torch.cuda.Stream object for it takes 2.9 us, this 0.3, and a small
    call's kernel is done in 5."""
    if stream is not None:
        return stream.cuda_stream or None
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None


def _elsewhere(stream) -> bool:
    """Whether `stream` is given and not the current one: a call that allocates goes through _on_stream then."""
    return stream is not None and stream.cuda_stream != (_stream_ptr() or 0)


def _on_stream(stream, call, *args, **kw):
    """A call that allocates, on another stream than the current one.  Workspaces and new results are blocks of `stream`: from the
    current stream's, a workspace dropped here could be in use again before `stream` has run the call, and a result could be written while the
    current stream still works on the block's last content.  The results belong to the caller's stream too: they are not used again before
    its work on them is done.  (The arguments are the caller's: `stream` has to run behind what made them, and they have to live until it is done.)"""
    import torch
    here = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        got = call(*args, **kw)
    for t in got if isinstance(got, tuple) else (got,):
        if t is not None:
            t.record_stream(here)
    return got


def stream_read(buf, out=None, stream=None):
    """csb_debug_stream_read on a device tensor (any dtype, size a multiple of 16 bytes)."""
    import torch
    if out is None and _elsewhere(stream):
        return _on_stream(stream, stream_read, buf)
    n = int(lib().csb_debug_stream_read_out_floats())
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=buf.device)
    assert out.numel() >= n and buf.is_contiguous()
    _check(lib().csb_debug_stream_read(_dptr(buf), buf.numel() * buf.element_size(), _dptr(out), _stream_ptr(stream)))
    return out


def project(W, br: int, bc: int, rate: float, out=None, stream=None):
    """csb_project on a device tensor W [rows][cols] (float32, rows may be strided): returns the
    pruned matrix (a new tensor, or `out`, which may be W itself)."""
    import torch
    if _elsewhere(stream):
        return _on_stream(stream, project, W, br, bc, rate, out)
    assert W.dim() == 2 and W.dtype == torch.float32 and W.stride(1) == 1
    rows, cols = W.shape
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.float32, device=W.device)
    assert out.shape == W.shape and out.dtype == torch.float32 and out.stride(1) == 1
    nb = int(lib().csb_project_workspace_bytes(rows, cols, br, bc))
    ws = torch.empty(max(nb, 256), dtype=torch.uint8, device=W.device)
    _check(lib().csb_project(W.data_ptr(), rows, cols, W.stride(0), br, bc, float(rate), out.data_ptr(), out.stride(0),
                             _dptr(ws), _stream_ptr(stream)))
    return out


def _val_type(dtype) -> int:
    """CSB_VAL_* of a torch dtype."""
    torch = sys.modules["torch"]
    if dtype is torch.bfloat16:
        return VAL_BF16
    if dtype is torch.float16:
        return VAL_F16
    assert dtype is torch.float32, f"expected a float32, float16 or bfloat16 tensor, got {dtype}"
    return VAL_F32


def _scratch(nbytes: int, device):
    """A workspace (torch's blocks are 512-byte aligned) of the current stream, which the call has to run on."""
    import torch
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


_DELTA_ARGS = struct.Struct("@6iq3P3q2P2q5PifPq")             # csb_delta_args, as ctypes lays it out


def _operands(floats, *others) -> int:
    """The current device, on which a call runs and all of its operands lie (None: not given).  The operators have no gradients: as torch does
    where it is given an `out`, they refuse numbers that ask for one while gradients are enabled, rather than return what has lost it."""
    assert floats[0].is_cuda
    torch = sys.modules["torch"]
    here = torch._C._cuda_getDevice()
    for t in floats:
        if t is not None:
            assert t.get_device() == here, "an operand that is not on the current device"
            assert not t.requires_grad or not torch.is_grad_enabled(), "no gradients here: an operand requires one (torch.no_grad() or detach())"
    for t in others:
        assert t is None or t.get_device() == here, "an operand that is not on the current device"
    return here


def _raw_stream(device: int) -> Optional[int]:
    """_stream_ptr() for callers that know the current device."""
    return sys.modules["torch"]._C._cuda_getCurrentRawStream(device) or None


def _ptr(t, dtype) -> int:
    """Address of a contiguous tensor that _operands has seen (None: 0)."""
    if t is None:
        return 0
    assert t.is_contiguous() and t.dtype is dtype, f"expected a contiguous {dtype} tensor"
    return t.data_ptr()


def _delta_rows(t, n, w, tokens):
    """Elements from one token to the next of [tokens, n, w]: (t, head, j) at t * ld + head * w + j."""
    if t.is_contiguous():
        return n * w
    ld, head, one = t.stride()
    assert (one == 1 or w == 1) and (head == w or n == 1), "heads of a token must be contiguous"
    return ld if tokens > 1 else max(ld, n * w)


def _delta(chunked, q, k, v, g, beta, scale, starts, lens, state, slots, state_out, out, stream):
    if _elsewhere(stream):
        return _on_stream(stream, _delta, chunked, q, k, v, g, beta, scale, starts, lens, state, slots, state_out, out, None)
    torch = sys.modules["torch"]
    T, HK, DK = shape = q.shape
    Tv, HV, DV = v.shape
    f32, typ = torch.float32, v.dtype
    assert T == Tv and k.shape == shape and g.shape == beta.shape == (T, HV)
    assert q.dtype is k.dtype is typ and g.dtype is beta.dtype is f32
    given = out
    here = _operands((q, k, v, g, beta, state, state_out if state_out is not state else None, out), starts, lens, slots)
    if out is None:
        out = torch.empty_like(v, memory_format=torch.contiguous_format)
    else:
        assert out.shape == v.shape and out.dtype is typ
    (ldg, one_g), (ldb, one_b) = g.stride(), beta.stride()
    assert one_g == one_b == 1 or HV == 1
    if T < 2:
        ldg = ldb = HV
    if starts is not None:
        N = starts.numel() - 1
    elif lens is not None:
        N = lens.numel()
    elif slots is not None:
        N = slots.numel()
    else:
        N = state.shape[0] if state is not None else 1
    assert (lens is None or lens.numel() == N) and (slots is None or slots.numel() == N)
    n_states = 0
    for t in (state,) if state_out is state else (state, state_out):
        if t is not None:
            assert t.shape[1:] == (HV, DK, DV) and n_states in (0, t.shape[0])
            n_states = t.shape[0]
    i32 = torch.int32
    args = (_val_type(typ), HK, HV, DK, DV, N, T, q.data_ptr(), k.data_ptr(), v.data_ptr(), _delta_rows(q, HK, DK, T),
            _delta_rows(k, HK, DK, T), _delta_rows(v, HV, DV, T), g.data_ptr(), beta.data_ptr(), ldg, ldb, _ptr(starts, i32),
            _ptr(lens, i32), _ptr(state, f32), _ptr(state_out, f32), _ptr(slots, i32), n_states, DK ** -0.5 if scale is None else scale, out.data_ptr(), _delta_rows(out, HV, DV, T))
    lib()
    raw = _DELTA_ARGS.pack(*args)
    if chunked:
        ws = _scratch(_raw_delta["workspace"](raw), v.device)
        rc = _raw_delta["chunked"](raw, ws.data_ptr() if ws is not None else None, _raw_stream(here))
    else:
        rc = _raw_delta["recurrent"](raw, _raw_stream(here))
    if rc:
        _check(rc)
    if state_out is not None:                                  # autograd may keep what has changed in place
        torch._C._increment_version((state_out,))
    if given is not None:
        torch._C._increment_version((given,))
    return out


_KEEP = object()


def delta_chunked(q, k, v, g, beta, scale=None, starts=None, lens=None, state=None, slots=None, state_out=_KEEP, out=None, stream=None):
    """csb_delta_chunked: the gated delta rule over whole prompts.  q, k [tokens, heads_k, dk], v [tokens, heads_v, dv] (one
    dtype: float32, float16 or bfloat16; rows of tokens may be strided), g (logarithm of the decay) and beta [tokens, heads_v]
    float32.  starts [n_seq + 1] int32: where the packed sequences start (None: all of one length, as many as lens, slots or
    states, or one).  lens [n_seq] int32: only that many tokens of each.  state [n_states, heads_v, dk, dv] float32, slots [n_seq] int32: each
    sequence's state in it (None: in order).  The last states go to state_out: `state` itself unless another tensor or
    None (not kept) is given.  scale: dk ** -0.5 unless given.  Returns out [tokens, heads_v, dv] (a new tensor, or `out`)."""
    return _delta(True, q, k, v, g, beta, scale, starts, lens, state, slots, state if state_out is _KEEP else state_out, out, stream)


def delta_recurrent(q, k, v, g, beta, scale=None, starts=None, lens=None, state=None, slots=None, state_out=_KEEP, out=None, stream=None):
    """csb_delta_recurrent: the same rule token by token, for the few tokens of a decoding step; arguments as delta_chunked."""
    return _delta(False, q, k, v, g, beta, scale, starts, lens, state, slots, state if state_out is _KEEP else state_out, out, stream)


def adapter_add(Y, X, A, B, ids, starts=None, scales=None, ranks=None, stream=None):
    """csb_adapter_add: Y[:, n] += scales[a] B[a] (A[a] X[:, n]) for the columns of every request, in place.  X [cols, batch], A [adapters,
    rank, cols] and B [adapters, rows, rank] of one dtype (float32, float16, bfloat16), Y [rows, batch] float32 (rows of X and Y may be
    strided).  ids [requests] int32: the adapter of each request, -1 for none; starts [requests + 1] int32: its columns (None: one
    each).  scales [adapters] float32, ranks [adapters] int32: factor and used ranks of an adapter.  Returns Y."""
    if _elsewhere(stream):
        return _on_stream(stream, adapter_add, Y, X, A, B, ids, starts, scales, ranks)
    torch = sys.modules["torch"]
    cols, batch = X.shape
    n, rank, A_cols = A.shape
    rows, Y_batch = Y.shape
    i32, f32, typ = torch.int32, torch.float32, X.dtype
    here = _operands((X, Y, A, B, scales), ids, starts, ranks)
    assert Y_batch == batch and Y.dtype is f32 and typ is A.dtype is B.dtype
    assert A_cols == cols and B.shape == (n, rows, rank)
    (ldx, one_x), (ldy, one_y) = X.stride(), Y.stride()
    assert batch < 2 or one_x == one_y == 1
    ldx, ldy = ldx if cols > 1 else batch, ldy if rows > 1 else batch          # (one row: its stride says nothing)
    segs = ids.numel()
    assert (starts is None or starts.numel() == segs + 1) and (scales is None or scales.numel() == n) and (ranks is None or ranks.numel() == n)
    L = lib()
    ws = torch.empty(max(L.csb_adapter_workspace_bytes(cols, batch, segs, rank), 256), dtype=torch.uint8, device=X.device)
    rc = L.csb_adapter_add(_val_type(typ), X.data_ptr(), ldx, Y.data_ptr(), ldy, rows, cols, batch, _ptr(A, typ), _ptr(B, typ),
                           n, rank, _ptr(ranks, i32), _ptr(scales, f32), segs, _ptr(starts, i32), _ptr(ids, i32), ws.data_ptr(),
                           _raw_stream(here))
    if rc:
        _check(rc)
    torch._C._increment_version((Y,))                          # (autograd may keep it as it was)
    return Y


def verify_drafts(p, q, drafts, u, r, counts=None, stream=None):
    """csb_verify_drafts: p [requests, drafts + 1, vocab] the target's probabilities, q [requests, drafts, vocab] the draft's (None: all
    of the mass on the drafted token) of one dtype (float32, float16, bfloat16); drafts [requests, n] int32, u [requests, n] and r [requests]
    float32 numbers in [0, 1); counts [requests] int32: drafts that a request brings (None: n).  Returns (tokens
    [requests, n + 1] int32: the accepted drafts, the token drawn behind them, -1; accepted [requests] int32)."""
    if _elsewhere(stream):
        return _on_stream(stream, verify_drafts, p, q, drafts, u, r, counts)
    torch = sys.modules["torch"]
    N, K1, V = p.shape
    K = K1 - 1
    i32, f32, typ, dev = torch.int32, torch.float32, p.dtype, p.device
    here = _operands((p, q, u, r), drafts, counts)

    def rows(t, n):
        before, ld, one = t.stride()
        assert one == 1 or V == 1
        if n < 2:
            ld = max(V, before)
        assert N < 2 or before == n * ld, "rows of the requests must follow each other at one stride"
        return ld
    assert drafts.shape == u.shape == (N, K) and r.numel() == N and (counts is None or counts.numel() == N)
    ldq = 0
    if q is not None and K:
        assert q.shape == (N, K, V) and q.dtype is typ
        ldq = rows(q, K)
    tokens = torch.empty((N, K1), dtype=i32, device=dev)
    accepted = torch.empty(N, dtype=i32, device=dev)
    L = lib()
    ws = torch.empty(max(L.csb_verify_workspace_bytes(N, V), 256), dtype=torch.uint8, device=dev)
    rc = L.csb_verify_drafts(_val_type(typ), p.data_ptr(), rows(p, K1), q.data_ptr() if ldq else None, ldq, _ptr(drafts, i32), _ptr(u, f32),
                             _ptr(r, f32), _ptr(counts, i32), N, K, V, tokens.data_ptr(), accepted.data_ptr(), ws.data_ptr(), _raw_stream(here))
    if rc:
        _check(rc)
    return tokens, accepted


def _rows(t, tokens, width) -> int:
    """Elements from one token to the next of [tokens, width]."""
    ld, one = t.stride()
    assert one == 1 or width == 1, "a token's entries must be contiguous"
    return ld if tokens > 1 else width


def _sequences(starts, lens, slots, state) -> int:
    """How many packed sequences a call has."""
    if starts is not None:
        n = starts.numel() - 1
    elif lens is not None:
        n = lens.numel()
    elif slots is not None:
        n = slots.numel()
    else:
        n = state.shape[0] if state is not None else 1
    assert (lens is None or lens.numel() == n) and (slots is None or slots.numel() == n)
    return n


def _states(state, state_out, shape) -> int:
    """How many states a call's tensors have room for."""
    n = 0
    for t in (state,) if state_out is state else (state, state_out):
        if t is not None:
            assert t.shape[1:] == shape and n in (0, t.shape[0])
            n = t.shape[0]
    return n


def _changed(*tensors):
    """Autograd may keep what has changed in place."""
    torch = sys.modules["torch"]
    for t in tensors:
        if t is not None:
            torch._C._increment_version((t,))


_CONV_ARGS = struct.Struct("@6iqPq8Pq")                       # csb_conv_args and csb_scan_args, as ctypes lays them out
_SCAN_ARGS = struct.Struct("@6iq5P5q8P2iPq")


def short_conv(x, weight, bias=None, silu=True, starts=None, lens=None, state=None, slots=None, state_out=_KEEP, out=None, stream=None):
    """csb_short_conv: the short causal convolution of a recurrent layer, channel by channel, and its activation.  x [tokens, channels]
    (float32, float16 or bfloat16; rows may be strided), weight [channels, width] (the last column is the token's own) and bias [channels]
    float32.  starts, lens and slots as delta_chunked; state [n_states, width - 1, channels] of x's dtype: the inputs before each sequence,
    oldest first.  The last inputs go to state_out: `state` itself unless another tensor or None (not kept) is given.  Returns out [tokens, channels]
    (a new tensor, or `out`, which must not overlap x)."""
    if state_out is _KEEP:
        state_out = state
    if _elsewhere(stream):
        return _on_stream(stream, short_conv, x, weight, bias, silu, starts, lens, state, slots, state_out, out)
    torch = sys.modules["torch"]
    T, CH = x.shape
    CW, W = weight.shape
    f32, i32, typ, given = torch.float32, torch.int32, x.dtype, out
    here = _operands((x, weight, bias, state, state_out if state_out is not state else None, out), starts, lens, slots)
    assert CW == CH and (bias is None or bias.numel() == CH)
    if out is None:
        out = torch.empty((T, CH), dtype=typ, device=x.device)
    else:
        assert out.shape == x.shape and out.dtype is typ
    N = _sequences(starts, lens, slots, state)
    n_states = _states(state, state_out, (W - 1, CH))
    lib()
    raw = _CONV_ARGS.pack(_val_type(typ), CH, W, bool(silu), N, n_states, T, x.data_ptr(), _rows(x, T, CH), _ptr(weight, f32), _ptr(bias, f32),
                          _ptr(starts, i32), _ptr(lens, i32), _ptr(state, typ), _ptr(state_out, typ), _ptr(slots, i32), out.data_ptr(),
                          _rows(out, T, CH))
    rc = _raw["csb_short_conv"](raw, _raw_stream(here))
    if rc:
        _check(rc)
    _changed(state_out, given)
    return out


def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, starts=None, lens=None, state=None, slots=None, state_out=_KEEP,
                   out=None, stream=None):
    """csb_selective_scan: the selective state space scan, for whole prompts and for the few tokens of a decoding step.  x, dt and z [tokens, channels],
    B and C [tokens, groups, n] of one dtype (float32, float16, bfloat16; rows of tokens may be strided); A [channels, n], D and dt_bias
    [channels] float32.  A token's step is ln(1 + e^(dt + dt_bias)), or dt + dt_bias without `softplus`; z: the gate (None: none).  starts, lens and slots as
    delta_chunked; state [n_states, channels, n] float32, the last states go to state_out: `state` itself unless another tensor or None (not
    kept) is given.  Returns out [tokens, channels] (a new tensor, or `out`, which may be x, dt or z)."""
    if state_out is _KEEP:
        state_out = state
    if _elsewhere(stream):
        return _on_stream(stream, selective_scan, x, dt, A, B, C, D, z, dt_bias, softplus, starts, lens, state, slots, state_out, out)
    torch = sys.modules["torch"]
    T, CH = shape = x.shape
    _, G, n = B.shape
    f32, i32, typ, given = torch.float32, torch.int32, x.dtype, out
    here = _operands((x, dt, A, B, C, D, z, dt_bias, state, state_out if state_out is not state else None, out), starts, lens, slots)
    assert dt.shape == shape and B.shape == C.shape == (T, G, n) and A.shape == (CH, n) and (z is None or z.shape == shape)
    assert dt.dtype is B.dtype is C.dtype is typ and (z is None or z.dtype is typ)
    assert (D is None or D.numel() == CH) and (dt_bias is None or dt_bias.numel() == CH)
    if out is None:
        out = torch.empty((T, CH), dtype=typ, device=x.device)
    else:
        assert out.shape == shape and out.dtype is typ
    N = _sequences(starts, lens, slots, state)
    n_states = _states(state, state_out, (CH, n))
    lib()
    raw = _SCAN_ARGS.pack(_val_type(typ), CH, G, n, bool(softplus), N, T, x.data_ptr(), dt.data_ptr(), z.data_ptr() if z is not None else 0,
                          B.data_ptr(), C.data_ptr(), _rows(x, T, CH), _rows(dt, T, CH), _rows(z, T, CH) if z is not None else 0,
                          _delta_rows(B, G, n, T), _delta_rows(C, G, n, T), _ptr(A, f32), _ptr(D, f32), _ptr(dt_bias, f32), _ptr(starts, i32),
                          _ptr(lens, i32), _ptr(state, f32), _ptr(state_out, f32), _ptr(slots, i32), n_states, 0, out.data_ptr(),
                          _rows(out, T, CH))
    ws = _scratch(_raw["csb_scan_workspace_bytes"](raw), x.device)
    rc = _raw["csb_selective_scan"](raw, ws.data_ptr() if ws is not None else None, _raw_stream(here))
    if rc:
        _check(rc)
    _changed(state_out, given)
    return out


_NORM_ARGS = struct.Struct("@q6i2f" + "Pq2i" * 5 + "5P")       # csb_norm_args, as ctypes lays it out
_NORMS = {None: 0, "rms": 1, "mean": 2}
_GATES = {"silu": 0, "sigmoid": 1}


def _order(t, shape):
    """A csb_norm_operand of [tokens, width]: rows or columns (a transposed view) by its strides."""
    if t is None:
        return 0, 0, 0, 0
    assert t.shape == shape
    (a, b), (tokens, width) = t.stride(), shape
    if b == 1 or width == 1:
        return t.data_ptr(), a if tokens > 1 else width, _val_type(t.dtype), 0
    assert a == 1 or tokens == 1, "entries of a token, or of all tokens at one place, must be contiguous"
    return t.data_ptr(), b, _val_type(t.dtype), 1


def block_norm(y=None, gate=None, x=None, after=None, after_weight=None, after_bias=None, groups=1, gate_kind="silu", gate_first=False, scale=1.0,
               scales=None, before=None, before_weight=None, before_bias=None, eps=1e-5, out=None, normed=None, stream=None):
    """csb_block_norm: norms around a block.  y [tokens, width] is the block's output, x the residual stream (one of them may be None), gate
    a gate; float32, float16 or bfloat16, each by itself, row by row or transposed views of column by column (a product's operands: Y.t()).
        p = norm_after(y), times act(gate) behind it, or before it with `gate_first`;  r = x + scale scales p;  n = norm_before(r)
    after, before: None, "rms" or "mean" (with the mean taken off), their weights and biases and scales [width] float32 (None: ones, zeros).
    groups: norm_after is over that many equal parts of a token.  gate_kind: "silu" or "sigmoid".  Returns (r, n): new tensors of x's dtype (y's without x)
    or `out` and `normed`; n is None without a norm before, r is x itself where there is no y and no `out`."""
    if _elsewhere(stream):
        return _on_stream(stream, block_norm, y, gate, x, after, after_weight, after_bias, groups, gate_kind, gate_first, scale, scales, before,
                          before_weight, before_bias, eps, out, normed)
    torch = sys.modules["torch"]
    main = x if x is not None else y
    T, W = shape = main.shape
    f32 = torch.float32
    factors = (after_weight, after_bias, scales, before_weight, before_bias)
    here = _operands((main, y, gate, *factors, out, normed))
    for w in factors:
        assert w is None or w.numel() == W
    assert before is not None or normed is None
    given, given_n, r = out, normed, out
    if out is None:
        if y is None and before is not None:
            r = x
        else:
            r = out = torch.empty((T, W), dtype=main.dtype, device=main.device)
    if before is not None and normed is None:
        normed = torch.empty((T, W), dtype=main.dtype, device=main.device)
    lib()
    raw = _NORM_ARGS.pack(T, W, groups, _NORMS[after], _NORMS[before], _GATES[gate_kind], bool(gate_first), scale, eps, *_order(y, shape), *_order(gate, shape),
                          *_order(x, shape), *_order(out, shape), *_order(normed, shape), *(_ptr(w, f32) for w in factors))
    rc = _raw["csb_block_norm"](raw, _raw_stream(here))
    if rc:
        _check(rc)
    _changed(given, given_n)
    return r, normed


def sample(logits, r=None, temperature=None, top_k=None, top_p=None, min_p=None, probs=False, stream=None):
    """csb_sample: the next token of every row of logits [rows, vocab] (float32, float16 or bfloat16; rows may be strided) from r [rows] float32, numbers
    in [0, 1).  temperature (0: the largest logit), top_p, min_p [rows] float32 and top_k [rows] int32 (None: 1, and all).  Returns tokens [rows]
    int32; with `probs` (tokens, the distribution that they are drawn from [rows, vocab] of logits' dtype, what verify_drafts takes); with r None that alone.
    probs may be a tensor that the distribution is written to (logits itself among them)."""
    if _elsewhere(stream):
        return _on_stream(stream, sample, logits, r, temperature, top_k, top_p, min_p, probs)
    torch = sys.modules["torch"]
    R, V = logits.shape
    i32, f32, typ, dev = torch.int32, torch.float32, logits.dtype, logits.device
    given = None if isinstance(probs, bool) else probs
    here = _operands((logits, r, temperature, top_p, min_p, given if given is not logits else None), top_k)
    for t in (r, temperature, top_k, top_p, min_p):
        assert t is None or t.numel() == R
    assert r is not None or probs is not False, "neither tokens nor their distribution"
    dist = given
    if given is not None:
        assert given.shape == logits.shape and given.dtype is typ
    elif probs:
        dist = torch.empty((R, V), dtype=typ, device=dev)
    tokens = torch.empty(R, dtype=i32, device=dev) if r is not None else None
    L = lib()
    ws = _scratch(L.csb_sample_workspace_bytes(R, V), dev)
    rc = L.csb_sample(_val_type(typ), logits.data_ptr(), _rows(logits, R, V), _ptr(temperature, f32), _ptr(top_k, i32), _ptr(top_p, f32), _ptr(min_p, f32),
                      _ptr(r, f32), R, V, _ptr(tokens, i32), dist.data_ptr() if dist is not None else None, _rows(dist, R, V) if dist is not None else 0,
                      ws.data_ptr() if ws is not None else None, _raw_stream(here))
    if rc:
        _check(rc)
    _changed(given)
    return tokens if dist is None else dist if tokens is None else (tokens, dist)


class CsbMatrix:
    """Owns one csb_matrix handle and (optionally) the torch buffer holding its device image."""

    def __init__(self, dense: np.ndarray, br: int, bc: int, ld: Optional[int] = None):
        dense = np.ascontiguousarray(dense, dtype=np.float32)
        rows, cols = dense.shape
        self._h = C.c_void_p()
        _check(lib().csb_pack(dense.ctypes.data, rows, cols, cols if ld is None else ld, br, bc, C.byref(self._h)))
        self.rows, self.cols, self.br, self.bc = rows, cols, br, bc
        self.d_buf = None
        self.d_ws = None
        self.stats = None

    @property
    def handle(self):
        return self._h

    def view(self):
        v = csb_view()
        _check(lib().csb_view_get(self._h, C.byref(v)))
        nb = v.nbr * v.nbc

        def arr(p, n, dt):
            return np.ctypeslib.as_array(p, shape=(n,)).astype(dt, copy=True) if n else np.zeros(0, dt)
        return dict(rows=v.rows, cols=v.cols, br=v.br, bc=v.bc, nbr=v.nbr, nbc=v.nbc, nnz=v.nnz,
                    nrows=arr(v.nrows, nb, np.int32), ncols=arr(v.ncols, nb, np.int32),
                    rowidx=arr(v.rowidx, v.n_rowidx, np.uint16), colidx=arr(v.colidx, v.n_colidx, np.uint16),
                    val=arr(v.val, v.nnz, np.float32),
                    val_off=arr(v.val_off, nb + 1, np.int64), row_off=arr(v.row_off, nb + 1, np.int64),
                    col_off=arr(v.col_off, nb + 1, np.int64))

    def unpack(self) -> np.ndarray:
        out = np.empty((self.rows, self.cols), np.float32)
        _check(lib().csb_unpack(self._h, out.ctypes.data, self.cols))
        return out

    def sharing_model(self, P: int = 4, Q: int = 4, K: int = 4, L: int = 4) -> dict:
        """csb_sharing_model: PE utilisation of the paper's own engine schedule on this matrix."""
        st = csb_sharing_stats()
        _check(lib().csb_sharing_model(self._h, P, Q, K, L, C.byref(st)))
        return {k: getattr(st, k) for k, _ in csb_sharing_stats._fields_}

    def set_value_format(self, fmt: int):
        """csb_set_value_format: VAL_F32 / VAL_F16 / VAL_BF16; plan and upload again afterwards."""
        _check(lib().csb_set_value_format(self._h, fmt))
        self.d_buf = None
        return self

    def value_format(self) -> int:
        return int(lib().csb_value_format(self._h))

    def plan(self, n_chunks: int = 0, mode: int = 0):
        st = csb_plan_stats()
        _check(lib().csb_plan_ex(self._h, n_chunks, mode, C.byref(st)))
        self.stats = {k: getattr(st, k) for k, _ in csb_plan_stats._fields_}
        return self.stats

    def plan_rows(self, n_workgroups: int = 0, min_rounds: int = 0):
        """csb_plan_rows: the row-owned mat-vec layout with its parameters spelled out."""
        st = csb_plan_stats()
        _check(lib().csb_plan_rows(self._h, n_workgroups, min_rounds, C.byref(st)))
        self.stats = {k: getattr(st, k) for k, _ in csb_plan_stats._fields_}
        self.d_buf = None
        return self.stats

    def plan_stats(self):
        """csb_plan_stats_get: the statistics of the current plan."""
        st = csb_plan_stats()
        _check(lib().csb_plan_stats_get(self._h, C.byref(st)))
        return {k: getattr(st, k) for k, _ in csb_plan_stats._fields_}

    def status(self, stream=None) -> int:
        """csb_status: non-zero if a merge of shared row tiles gave up since the last check."""
        v = C.c_int32(0)
        _check(lib().csb_status(self._h, _stream_ptr(stream), C.byref(v)))
        return int(v.value)

    def validate(self):
        _check(lib().csb_plan_validate(self._h))

    def device_bytes(self) -> int:
        return int(lib().csb_device_bytes(self._h))

    def workspace_bytes(self, batch: int = 1) -> int:
        return int(lib().csb_workspace_bytes(self._h, batch))

    def upload(self, device="cuda", stream=None):
        """Allocate the image buffer with torch and copy the planned image into it."""
        import torch
        n = self.device_bytes()
        self.d_buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
        base = self.d_buf.data_ptr()
        self._d_ptr = (base + 255) // 256 * 256
        _check(lib().csb_upload(self._h, self._d_ptr, n, _stream_ptr(stream)))
        return self

    def spmv(self, x, y=None, stream=None):
        import torch
        if (y is None or self.d_ws is None) and _elsewhere(stream):
            return _on_stream(stream, self.spmv, x, y)
        if y is None:
            y = torch.empty(self.rows, dtype=torch.float32, device=x.device)
        ws = self._workspace(1, x.device)
        _check(lib().csb_spmv(self._h, _dptr(x, _f32()), _dptr(y, _f32()), _dptr(ws), _stream_ptr(stream)))
        return y

    def spmv_static(self, x, y=None, stream=None):
        """csb_spmv_static: csb_spmv with the library's built-in buffer in place of a workspace."""
        import torch
        if y is None and _elsewhere(stream):
            return _on_stream(stream, self.spmv_static, x)
        if y is None:
            y = torch.empty(self.rows, dtype=torch.float32, device=x.device)
        _check(lib().csb_spmv_static(self._h, _dptr(x, _f32()), _dptr(y, _f32()), _stream_ptr(stream)))
        return y

    def spmv_stamps(self, x, y=None, stream=None):
        """csb_debug_spmv_stamps: returns (y, stamps).  Row-owned layout: int64 [n_workgroups, 16, 8]
        (per wavefront: start, vector staged, first unit landed, same, groups done, after the
        barrier, end; 100 MHz clock).  Tile-based layout: [n_chunks, 8 + 3*16] shader clocks."""
        import torch
        if _elsewhere(stream):
            return _on_stream(stream, self.spmv_stamps, x, y)
        if y is None:
            y = torch.empty(self.rows, dtype=torch.float32, device=x.device)
        n = int(lib().csb_debug_stamp_count(self._h))
        st = torch.zeros(n, dtype=torch.int64, device=x.device)
        ws = self._workspace(1, x.device)
        _check(lib().csb_debug_spmv_stamps(self._h, _dptr(x, _f32()), _dptr(y, _f32()), _dptr(ws), _dptr(st), _stream_ptr(stream)))
        if getattr(self, "stats", None) and self.stats.get("row_owned") == 1:
            return y, st.view(-1, 16, 8)
        return y, st.view(-1, 8 + 3 * 16)

    def spmm(self, X, Y=None, stream=None):
        import torch
        if Y is None and _elsewhere(stream):
            return _on_stream(stream, self.spmm, X)
        cols, batch = X.shape
        if Y is None:
            Y = torch.empty((self.rows, batch), dtype=torch.float32, device=X.device)
        # rows may be strided views ([cols][ldx], [rows][ldy]); the batch index must be contiguous
        (ldx, one_x), (ldy, one_y) = X.stride(), Y.stride()
        assert X.is_cuda and Y.is_cuda and one_x == 1 and one_y == 1
        assert X.dtype is torch.float32 and Y.dtype is torch.float32
        _check(lib().csb_spmm(self._h, X.data_ptr(), ldx, Y.data_ptr(), ldy, batch, None, _stream_ptr(stream)))   # (no workspace: csb_spmm reads none)
        return Y

    def spmm_bfloat(self, Xb, Y=None, stream=None):
        """Xb: [cols, batch] torch.bfloat16 cuda (rows may be strided, the batch contiguous)."""
        import torch
        if Y is None and _elsewhere(stream):
            return _on_stream(stream, self.spmm_bfloat, Xb)
        cols, batch = Xb.shape
        if Y is None:
            Y = torch.empty((self.rows, batch), dtype=torch.float32, device=Xb.device)
        (ldx, one_x), (ldy, one_y) = Xb.stride(), Y.stride()
        assert Xb.is_cuda and Y.is_cuda and Xb.dtype is torch.bfloat16 and one_x == 1 and one_y == 1
        _check(lib().csb_spmm_bfloat(self._h, Xb.data_ptr(), ldx, Y.data_ptr(), ldy, batch, _stream_ptr(stream)))
        return Y

    def spmm_half(self, Xh, Y=None, stream=None):
        """Xh: [cols, batch] torch.float16 cuda (rows may be strided, the batch contiguous)."""
        import torch
        if Y is None and _elsewhere(stream):
            return _on_stream(stream, self.spmm_half, Xh)
        cols, batch = Xh.shape
        if Y is None:
            Y = torch.empty((self.rows, batch), dtype=torch.float32, device=Xh.device)
        (ldx, one_x), (ldy, one_y) = Xh.stride(), Y.stride()
        assert Xh.is_cuda and Y.is_cuda and Xh.dtype is torch.float16 and one_x == 1 and one_y == 1
        _check(lib().csb_spmm_half(self._h, Xh.data_ptr(), ldx, Y.data_ptr(), ldy, batch, _stream_ptr(stream)))
        return Y

    def _workspace(self, batch, device):
        import torch
        need = self.workspace_bytes(batch)
        if need == 0:
            return None
        if self.d_ws is None or self.d_ws.numel() * 4 < need:
            self.d_ws = torch.empty((need + 3) // 4, dtype=torch.float32, device=device)
        return self.d_ws

    def close(self):
        if self._h:
            lib().csb_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class CsbRnn:
    """csb_rnn handle; keeps its matrices and bias tensors alive."""

    def __init__(self, cell: int, input: int, hidden: int, W: Sequence[CsbMatrix], bias=None,
                 proj: int = 0, Wp: Optional[Sequence[CsbMatrix]] = None):
        """cell CELL_LSTM / CELL_GRU / CELL_LIGRU: csb_rnn_create.  cell CELL_LSTMP:
        csb_rnn_create_lstmp with the projection width `proj` and the projection matrices `Wp`.
        cell CELL_GRU_RB: csb_rnn_create_gru_rb, `W` = the Wa matrices, `Wp` = the Un matrices."""
        self.cell, self.input, self.hidden, self.W = cell, input, hidden, list(W)
        self.proj, self.Wp = proj, (list(Wp) if Wp is not None else [])
        self.bias = list(bias) if bias is not None else None
        L = len(self.W)
        Wv = (C.c_void_p * L)(*[w.handle for w in self.W])
        Bp = None
        if self.bias is not None:
            Bp = (C.c_void_p * L)(*[_dptr(b, _f32()) for b in self.bias])
        self._h = C.c_void_p()
        if cell == CELL_LSTMP:
            assert proj > 0 and len(self.Wp) == L
            Pv = (C.c_void_p * L)(*[w.handle for w in self.Wp])
            _check(lib().csb_rnn_create_lstmp(L, input, hidden, proj, Wv, Pv, Bp, C.byref(self._h)))
        elif cell == CELL_GRU_RB:
            assert len(self.Wp) == L
            Pv = (C.c_void_p * L)(*[w.handle for w in self.Wp])
            _check(lib().csb_rnn_create_gru_rb(L, input, hidden, Wv, Pv, Bp, C.byref(self._h)))
        else:
            _check(lib().csb_rnn_create(cell, L, input, hidden, Wv, Bp, C.byref(self._h)))
        self.n_layers = L
        self._ws = None

    def workspace_bytes(self, batch: int, T: int) -> int:
        return int(lib().csb_rnn_workspace_bytes(self._h, batch, T))

    def stats(self):
        st = csb_rnn_plan_stats()
        _check(lib().csb_rnn_stats(self._h, C.byref(st)))
        return {k: getattr(st, k) for k, _ in csb_rnn_plan_stats._fields_ if k != "reserved"}

    def device_bytes(self) -> int:
        return int(lib().csb_rnn_device_bytes(self._h))

    def set_poll_limit(self, polls: int):
        _check(lib().csb_rnn_set_poll_limit(self._h, polls))
        return self

    def status(self, stream=None) -> int:
        """csb_rnn_status: non-zero if a wait inside the resident kernel gave up since the last check."""
        v = C.c_int32(0)
        _check(lib().csb_rnn_status(self._h, _stream_ptr(stream), C.byref(v)))
        return int(v.value)

    def plan_resident(self, batch: int):
        """Lay the resident kernel out for batches of this size (1: one sequence, as created);
        upload() afterwards."""
        _check(lib().csb_rnn_plan_resident(self._h, batch))
        self._d_img = None
        return self

    def upload(self, device="cuda", stream=None):
        """Upload the resident layout; without it forward() streams the matrices."""
        import torch
        n = self.device_bytes()
        if n == 0:
            raise CsbError(-4, "model has no resident layout")
        self._d_img = torch.empty(n + 256, dtype=torch.uint8, device=device)
        ptr = (self._d_img.data_ptr() + 255) // 256 * 256
        _check(lib().csb_rnn_upload(self._h, ptr, n, _stream_ptr(stream)))
        return self

    def forward(self, x, h0=None, c0=None, want_hseq=True, stream=None):
        """x: [T, B, I] float32 cuda.  Returns (hseq or None, hT, cT or None)."""
        import torch
        if _elsewhere(stream):
            return _on_stream(stream, self.forward, x, h0, c0, want_hseq)
        T, B, I = x.shape
        dev = x.device
        need = self.workspace_bytes(B, T)
        if self._ws is None or self._ws.numel() * 4 < need:
            self._ws = torch.empty((need + 3) // 4 + 64, dtype=torch.float32, device=dev)
        hs = self.proj if self.cell == CELL_LSTMP else self.hidden        # width of the state h
        hseq = torch.empty((T, B, hs), dtype=torch.float32, device=dev) if want_hseq else None
        hT = torch.empty((self.n_layers, B, hs), dtype=torch.float32, device=dev)
        cT = (torch.empty((self.n_layers, B, self.hidden), dtype=torch.float32, device=dev)
              if self.cell in (CELL_LSTM, CELL_LSTMP) else None)
        f32 = torch.float32
        _check(lib().csb_rnn_forward(self._h, _dptr(x, f32), _dptr(h0, f32), _dptr(c0, f32), _dptr(hseq, f32), _dptr(hT, f32), _dptr(cT, f32),
                                     T, B, self._ws.data_ptr(), _stream_ptr(stream)))
        return hseq, hT, cT

    def forward_into(self, x, h0, c0, hseq, hT, cT, stream=None):
        """csb_rnn_forward into the caller's output tensors (hseq, cT may be None)."""
        import torch
        T, B, I = x.shape
        need = self.workspace_bytes(B, T)
        if self._ws is None or self._ws.numel() * 4 < need:
            if _elsewhere(stream):
                return _on_stream(stream, self.forward_into, x, h0, c0, hseq, hT, cT)
            self._ws = torch.empty((need + 3) // 4 + 64, dtype=torch.float32, device=x.device)
        f32 = torch.float32
        _check(lib().csb_rnn_forward(self._h, _dptr(x, f32), _dptr(h0, f32), _dptr(c0, f32), _dptr(hseq, f32), _dptr(hT, f32),
                                     _dptr(cT, f32), T, B, self._ws.data_ptr(), _stream_ptr(stream)))

    def close(self):
        if self._h:
            lib().csb_rnn_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
