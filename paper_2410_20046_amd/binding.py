"""Thin ctypes binding of libdqrm.so: argument marshalling only.

Every function has the name of the C entry point it calls (``include/dqrm.h``)
and passes device pointers of torch tensors plus the current HIP stream.  No
step of the path runs in Python or in torch; torch only owns device memory and
streams.  There is no CPU fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

import numpy as np
import torch

from . import build as _build

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_WORKSPACE_TOO_SMALL = -3
ERR_INDEX_OUT_OF_RANGE = -4
ERR_HIP = -5
ERR_CAPACITY = -6
ERR_BAD_OFFSETS = -7
ERR_SCRATCH_LIMIT = -8
_NAMES = {0: "OK", -1: "INVALID_ARG", -2: "UNSUPPORTED", -3: "WORKSPACE_TOO_SMALL", -4: "INDEX_OUT_OF_RANGE",
          -5: "HIP_ERROR", -6: "CAPACITY", -7: "BAD_OFFSETS", -8: "SCRATCH_LIMIT"}

FWD_MASTER = 0
FWD_PACKED = 1
SEG_CHUNK = 32
MAX_TABLE_LOOKUPS = 65536
MAX_TABLES = 1024
MAX_DIM = 256
NOALLOC_SCRATCH_BYTES = 8 << 20

EXPORTS = ("dqrm_find_scale", "dqrm_pack_int4", "dqrm_embbag_fwd", "dqrm_embbag_bwd_workspace_bytes",
           "dqrm_embbag_bwd", "dqrm_embbag_bwd_noalloc", "dqrm_dedupe", "dqrm_dedupe_multi", "dqrm_segment_sum", "dqrm_segment_sum_multi",
           "dqrm_grad_quant_int8", "dqrm_grad_quant_int8_multi",
           "dqrm_sparse_update", "dqrm_sparse_merge_workspace_bytes", "dqrm_sparse_merge", "dqrm_sparse_update_sums",
           "dqrm_quant_update", "dqrm_fwd_bwd_step", "dqrm_dense_workspace_bytes", "dqrm_dense_step",
           "dqrm_dense_param_count", "dqrm_dense_step_quant", "dqrm_mxfp4_quant_workspace_bytes", "dqrm_mxfp4_quant",
           "dqrm_mxfp4_dequant", "dqrm_mxfp4_matmul_workspace_bytes", "dqrm_mxfp4_matmul", "dqrm_mxfp4_linear_workspace_bytes",
           "dqrm_mxfp4_linear", "dqrm_layernorm_fwd", "dqrm_layernorm_bwd_workspace_bytes", "dqrm_layernorm_bwd",
           "dqrm_residual_norm_fwd", "dqrm_residual_norm_bwd_workspace_bytes", "dqrm_residual_norm_bwd",
           "dqrm_softmax_xent_fwd_workspace_bytes", "dqrm_softmax_xent_fwd", "dqrm_softmax_xent_bwd_workspace_bytes", "dqrm_softmax_xent_bwd",
           "dqrm_grad_workspace_bytes", "dqrm_grad_norm", "dqrm_grad_scale", "dqrm_grad_clip", "dqrm_check_status", "dqrm_last_hip_error", "dqrm_version")


class DqrmError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: DQRM_ERR_{_NAMES.get(code, code)}" + (f" ({detail})" if detail else ""))


class dqrm_tables_t(C.Structure):
    _fields_ = [("num_tables", C.c_int32), ("dim", C.c_int32), ("row_offsets_host", C.c_void_p),
                ("row_offsets_dev", C.c_void_p), ("master", C.c_void_p), ("packed", C.c_void_p),
                ("w_scale", C.c_void_p)]


class dqrm_sparse_block_t(C.Structure):
    _fields_ = [("uniq_rows", C.c_void_p), ("table_uniq_offsets", C.c_void_p), ("gq", C.c_void_p),
                ("capacity", C.c_int64)]


class dqrm_dedupe_batch_t(C.Structure):
    _fields_ = [("indices", C.c_void_p), ("offsets", C.c_void_p), ("num_indices", C.c_int64),
                ("sorted_pos", C.c_void_p), ("uniq_rows", C.c_void_p), ("seg_offsets", C.c_void_p),
                ("table_uniq_offsets", C.c_void_p), ("num_unique", C.c_void_p), ("workspace", C.c_void_p),
                ("max_table_lookups", C.c_int32)]


MAX_DEDUPE_BATCHES = 8


class dqrm_segsum_batch_t(C.Structure):
    _fields_ = [("num_indices", C.c_int64), ("grad_out", C.c_void_p), ("values", C.c_void_p), ("g_absmax", C.c_void_p),
                ("workspace", C.c_void_p)]


class dqrm_quant_block_t(C.Structure):
    _fields_ = [("capacity", C.c_int64), ("values", C.c_void_p), ("table_uniq_offsets", C.c_void_p),
                ("g_absmax", C.c_void_p), ("gq", C.c_void_p), ("g_scale", C.c_void_p)]


class dqrm_dense_model_t(C.Structure):
    _fields_ = [("num_dense", C.c_int32), ("num_tables", C.c_int32), ("dim", C.c_int32), ("bot_layers", C.c_int32),
                ("bot_dims", C.c_void_p), ("bot_w", C.c_void_p), ("bot_b", C.c_void_p), ("top_layers", C.c_int32),
                ("top_dims", C.c_void_p), ("top_w", C.c_void_p), ("top_b", C.c_void_p)]


class dqrm_dense_quant_t(C.Structure):
    _fields_ = [("weight_bits", C.c_int32), ("grad_bits", C.c_int32), ("grad_error", C.c_void_p),
                ("grad_scale", C.c_void_p), ("grad_codes", C.c_void_p), ("grads", C.c_void_p), ("wq", C.c_void_p),
                ("grad_buffer", C.c_void_p), ("buffer_add", C.c_int32), ("buffer_update", C.c_int32)]


class dqrm_mxfp4_t(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p)]


class dqrm_residual_norm_t(C.Structure):
    _fields_ = [("post", C.c_int32), ("pre", C.c_int32), ("post_gamma", C.c_void_p), ("post_beta", C.c_void_p), ("gate", C.c_void_p),
                ("pre_gamma", C.c_void_p), ("pre_beta", C.c_void_p), ("res_scale", C.c_float), ("post_eps", C.c_float), ("pre_eps", C.c_float)]


class dqrm_grad_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("out", C.c_void_p), ("ld_out", C.c_int64),
                ("count", C.c_void_p), ("dtype", C.c_int32)]


NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
GRAD_NORM_2, GRAD_NORM_MAX = 0, 1
F32, BF16, F16 = 0, 1, 2
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """The loaded C-ABI library.  Builds it only if no built library is present."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if not os.path.exists(path):
            _build.build_library(force=True)
        L = C.CDLL(path)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        tp = C.POINTER(dqrm_tables_t)
        L.dqrm_find_scale.argtypes = [tp, vp]
        L.dqrm_pack_int4.argtypes = [tp, vp]
        L.dqrm_embbag_fwd.argtypes = [tp, vp, vp, i32, i64, i32, vp, vp, vp]
        L.dqrm_embbag_bwd_workspace_bytes.argtypes = [i32, i32, i32, i64]
        L.dqrm_embbag_bwd_workspace_bytes.restype = sz
        L.dqrm_embbag_bwd.argtypes = [tp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dqrm_embbag_bwd_noalloc.argtypes = [tp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.dqrm_embbag_bwd_noalloc.restype = i32
        L.dqrm_dedupe.argtypes = [tp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dqrm_dedupe_multi.argtypes = [tp, i32, i32, C.POINTER(dqrm_dedupe_batch_t), sz, vp]
        L.dqrm_dedupe_multi.restype = i32
        L.dqrm_segment_sum.argtypes = [tp, i32, i64, vp, vp, vp, vp, sz, vp]
        L.dqrm_segment_sum_multi.argtypes = [tp, i32, i32, C.POINTER(dqrm_segsum_batch_t), sz, vp]
        L.dqrm_segment_sum_multi.restype = i32
        L.dqrm_grad_quant_int8_multi.argtypes = [i32, i32, i32, C.POINTER(dqrm_quant_block_t), vp]
        L.dqrm_grad_quant_int8_multi.restype = i32
        L.dqrm_quant_update.argtypes = [tp, i64, i64, vp, vp, vp, vp, vp, vp, C.c_float, vp, sz, vp]
        L.dqrm_fwd_bwd_step.argtypes = [tp, vp, vp, i32, i64, i32, vp, vp, vp, C.c_float, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dqrm_fwd_bwd_step.restype = i32
        L.dqrm_grad_quant_int8.argtypes = [i32, i32, i64, vp, vp, vp, vp, vp, vp]
        L.dqrm_sparse_update.argtypes = [tp, i64, vp, vp, vp, vp, C.c_float, vp]
        L.dqrm_sparse_update_sums.argtypes = [tp, i64, vp, vp, vp, vp, C.c_float, vp]
        L.dqrm_sparse_update_sums.restype = i32
        L.dqrm_sparse_merge_workspace_bytes.argtypes = [i32, i32, i32, i64]
        L.dqrm_sparse_merge_workspace_bytes.restype = sz
        L.dqrm_sparse_merge.argtypes = [tp, i32, C.POINTER(dqrm_sparse_block_t), i64, vp, vp, vp, vp, vp, sz, vp]
        L.dqrm_sparse_merge.restype = i32
        dp = C.POINTER(dqrm_dense_model_t)
        L.dqrm_dense_workspace_bytes.argtypes = [dp, i32]
        L.dqrm_dense_workspace_bytes.restype = sz
        L.dqrm_dense_step.argtypes = [dp, i32, vp, vp, vp, C.c_float, vp, vp, vp, sz, vp]
        L.dqrm_dense_step.restype = i32
        L.dqrm_dense_param_count.argtypes = [dp]
        L.dqrm_dense_param_count.restype = i64
        L.dqrm_dense_step_quant.argtypes = [dp, C.POINTER(dqrm_dense_quant_t), i32, vp, vp, vp, C.c_float, vp, vp, vp,
                                            sz, vp]
        L.dqrm_dense_step_quant.restype = i32
        qp, f32 = C.POINTER(dqrm_mxfp4_t), C.c_float
        L.dqrm_mxfp4_quant.argtypes = [i32, i64, i64, vp, i64, vp, i64, qp, qp, vp, vp, sz, vp]
        L.dqrm_mxfp4_dequant.argtypes = [qp, i32, vp, i64, vp]
        L.dqrm_mxfp4_matmul.argtypes = [qp, qp, vp, i32, i32, vp, i64, vp, sz, vp]
        L.dqrm_mxfp4_linear.argtypes = [i32, i64, vp, i64, i32, vp, vp, f32, qp, vp, i32, vp, i64, vp, sz, vp]
        L.dqrm_layernorm_fwd.argtypes = [i32, i64, i64, vp, i64, vp, vp, f32, vp, i64, vp, vp, qp, vp]
        L.dqrm_layernorm_bwd.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        L.dqrm_mxfp4_quant_workspace_bytes.argtypes = L.dqrm_layernorm_bwd_workspace_bytes.argtypes = [i64, i64]
        L.dqrm_mxfp4_matmul_workspace_bytes.argtypes = L.dqrm_mxfp4_linear_workspace_bytes.argtypes = [i64, i64, i64]
        for n in ("quant", "matmul", "linear"):
            getattr(L, f"dqrm_mxfp4_{n}").restype = i32
            getattr(L, f"dqrm_mxfp4_{n}_workspace_bytes").restype = sz
        L.dqrm_mxfp4_dequant.restype = L.dqrm_layernorm_fwd.restype = L.dqrm_layernorm_bwd.restype = i32
        L.dqrm_layernorm_bwd_workspace_bytes.restype = sz
        np_, gp = C.POINTER(dqrm_residual_norm_t), C.POINTER(dqrm_grad_t)
        L.dqrm_residual_norm_fwd.argtypes = [i32, i64, i64, np_, vp, i64, vp, i64, vp, i64, vp, i64, vp, qp, vp]
        L.dqrm_residual_norm_bwd_workspace_bytes.argtypes = [i64, i64]
        L.dqrm_residual_norm_bwd.argtypes = [i32, i64, i64, np_] + [vp, i64] * 4 + [vp] + [vp, i64] * 2 + [vp, vp, sz, vp]
        L.dqrm_softmax_xent_fwd_workspace_bytes.argtypes = L.dqrm_softmax_xent_bwd_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.dqrm_softmax_xent_fwd.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, f32, vp, vp, vp, vp, sz, vp]
        L.dqrm_softmax_xent_bwd.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, f32, vp, vp, vp, vp, i64, vp, i64, vp, vp, sz, vp]
        L.dqrm_grad_workspace_bytes.argtypes = [gp, i32]
        L.dqrm_grad_norm.argtypes = [gp, i32, i32, vp, vp, vp, sz, vp]
        L.dqrm_grad_scale.argtypes = [gp, i32, vp, f32, vp]
        L.dqrm_grad_clip.argtypes = [gp, i32, i32, f32, vp, vp, vp, sz, vp]
        for n in ("residual_norm_fwd", "residual_norm_bwd", "softmax_xent_fwd", "softmax_xent_bwd", "grad_norm", "grad_scale", "grad_clip"):
            getattr(L, f"dqrm_{n}").restype = i32
        for n in ("residual_norm_bwd", "softmax_xent_fwd", "softmax_xent_bwd", "grad"):
            getattr(L, f"dqrm_{n}_workspace_bytes").restype = sz
        L.dqrm_check_status.argtypes = [vp, C.POINTER(i32), C.POINTER(i64)]
        for n in ("dqrm_find_scale", "dqrm_pack_int4", "dqrm_embbag_fwd", "dqrm_embbag_bwd", "dqrm_dedupe", "dqrm_segment_sum",
                  "dqrm_quant_update", "dqrm_grad_quant_int8", "dqrm_sparse_update", "dqrm_check_status"):
            getattr(L, n).restype = i32
        L.dqrm_last_hip_error.restype = C.c_char_p
        L.dqrm_version.restype = C.c_char_p
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "DQRM buffers must be contiguous"
    return t.data_ptr()


# the current stream's handle without making a Stream object (2.8 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, where: str) -> None:
    if rc != OK:
        detail = lib().dqrm_last_hip_error().decode() if rc == ERR_HIP else ""
        raise DqrmError(rc, where, detail)


class Tables:
    """Owns the device buffers of the embedding layer and the C descriptor."""

    def __init__(self, row_offsets: np.ndarray, dim: int, master: torch.Tensor, packed: Optional[torch.Tensor] = None,
                 w_scale: Optional[torch.Tensor] = None):
        self.row_offsets_host = np.ascontiguousarray(row_offsets, dtype=np.int64)
        self.T = len(self.row_offsets_host) - 1
        self.D = int(dim)
        self.R = int(self.row_offsets_host[-1])
        dev = master.device
        assert master.dtype == torch.float32 and tuple(master.shape) == (self.R, self.D)
        self.master = master
        self.packed = packed
        if packed is not None:
            assert packed.dtype == torch.uint8 and tuple(packed.shape) == (self.R, self.D // 2)
        self.w_scale = w_scale if w_scale is not None else torch.ones(self.T, dtype=torch.float32, device=dev)
        self.row_offsets_dev = torch.from_numpy(self.row_offsets_host).to(dev)
        self.c = dqrm_tables_t(self.T, self.D, self.row_offsets_host.ctypes.data, _ptr(self.row_offsets_dev),
                               _ptr(self.master), _ptr(self.packed), _ptr(self.w_scale))

    @property
    def ref(self):
        return C.byref(self.c)


def dqrm_version() -> str:
    return lib().dqrm_version().decode()


def dqrm_find_scale(tables: Tables, stream=None) -> None:
    _check(lib().dqrm_find_scale(tables.ref, _stream(stream)), "dqrm_find_scale")


def dqrm_pack_int4(tables: Tables, stream=None) -> None:
    _check(lib().dqrm_pack_int4(tables.ref, _stream(stream)), "dqrm_pack_int4")


def dqrm_embbag_fwd(tables: Tables, indices: torch.Tensor, offsets: torch.Tensor, batch: int, mode: int,
                    out: torch.Tensor, codes_dbg: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().dqrm_embbag_fwd(tables.ref, _ptr(indices), _ptr(offsets), batch, indices.numel(), mode, _ptr(out),
                                 _ptr(codes_dbg), _stream(stream)), "dqrm_embbag_fwd")


def dqrm_embbag_bwd_workspace_bytes(num_tables: int, dim: int, batch: int, num_indices: int) -> int:
    return int(lib().dqrm_embbag_bwd_workspace_bytes(num_tables, dim, batch, num_indices))


def dqrm_embbag_bwd(tables: Tables, indices: torch.Tensor, offsets: torch.Tensor, batch: int, grad_out: torch.Tensor,
                    sorted_pos: torch.Tensor, uniq_rows: torch.Tensor, seg_offsets: torch.Tensor,
                    table_uniq_offsets: torch.Tensor, num_unique: torch.Tensor, values: torch.Tensor,
                    g_absmax: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_embbag_bwd(tables.ref, _ptr(indices), _ptr(offsets), batch, indices.numel(), _ptr(grad_out),
                                 _ptr(sorted_pos), _ptr(uniq_rows), _ptr(seg_offsets), _ptr(table_uniq_offsets),
                                 _ptr(num_unique), _ptr(values), _ptr(g_absmax), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "dqrm_embbag_bwd")


def dqrm_embbag_bwd_noalloc(tables: Tables, indices: torch.Tensor, offsets: torch.Tensor, batch: int,
                            grad_out: torch.Tensor, sorted_pos: torch.Tensor, uniq_rows: torch.Tensor,
                            seg_offsets: torch.Tensor, table_uniq_offsets: torch.Tensor, num_unique: torch.Tensor,
                            values: torch.Tensor, g_absmax: torch.Tensor, stream=None) -> None:
    rc = lib().dqrm_embbag_bwd_noalloc(tables.ref, _ptr(indices), _ptr(offsets), batch, indices.numel(), _ptr(grad_out),
                                       _ptr(sorted_pos), _ptr(uniq_rows), _ptr(seg_offsets), _ptr(table_uniq_offsets),
                                       _ptr(num_unique), _ptr(values), _ptr(g_absmax), _stream(stream))
    if rc == ERR_SCRATCH_LIMIT:
        raise DqrmError(rc, "dqrm_embbag_bwd_noalloc", lib().dqrm_last_hip_error().decode())
    _check(rc, "dqrm_embbag_bwd_noalloc")


def dqrm_dedupe(tables: Tables, indices: torch.Tensor, offsets: torch.Tensor, batch: int, sorted_pos: torch.Tensor,
                uniq_rows: torch.Tensor, seg_offsets: torch.Tensor, table_uniq_offsets: torch.Tensor,
                num_unique: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_dedupe(tables.ref, _ptr(indices), _ptr(offsets), batch, indices.numel(), _ptr(sorted_pos),
                             _ptr(uniq_rows), _ptr(seg_offsets), _ptr(table_uniq_offsets), _ptr(num_unique),
                             _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "dqrm_dedupe")


def dqrm_dedupe_multi(tables: Tables, batch: int, batches, stream=None, max_table_lookups: int = 0) -> None:
    """``batches``: sequence of tuples (indices, offsets, sorted_pos, uniq_rows, seg_offsets, table_uniq_offsets,
    num_unique, workspace) of device tensors, one per batch (at most MAX_DEDUPE_BATCHES).  ``max_table_lookups``:
    the caller's bound on the lookups of any one table in any of the batches, 0 if none is known."""
    arr = (dqrm_dedupe_batch_t * len(batches))()
    ws_bytes = None
    for i, (ix, of, sp, ur, so, tuo, nu, ws) in enumerate(batches):
        arr[i] = dqrm_dedupe_batch_t(_ptr(ix), _ptr(of), ix.numel(), _ptr(sp), _ptr(ur), _ptr(so), _ptr(tuo), _ptr(nu),
                                     _ptr(ws), max_table_lookups)
        nb = ws.numel() * ws.element_size()
        ws_bytes = nb if ws_bytes is None else min(ws_bytes, nb)
    _check(lib().dqrm_dedupe_multi(tables.ref, batch, len(batches), arr, ws_bytes or 0, _stream(stream)),
           "dqrm_dedupe_multi")


def dqrm_segment_sum(tables: Tables, batch: int, num_indices: int, grad_out: torch.Tensor, values: torch.Tensor,
                     g_absmax: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_segment_sum(tables.ref, batch, num_indices, _ptr(grad_out), _ptr(values), _ptr(g_absmax),
                                  _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "dqrm_segment_sum")


def dqrm_segment_sum_multi(tables: Tables, batch: int, batches, stream=None) -> None:
    """``batches``: sequence of tuples (num_indices, grad_out, values, g_absmax or None, workspace) of device tensors,
    one per batch (at most MAX_DEDUPE_BATCHES)."""
    arr = (dqrm_segsum_batch_t * len(batches))()
    ws_bytes = None
    for i, (n, g, v, am, ws) in enumerate(batches):
        arr[i] = dqrm_segsum_batch_t(int(n), _ptr(g), _ptr(v), _ptr(am), _ptr(ws))
        nb = ws.numel() * ws.element_size()
        ws_bytes = nb if ws_bytes is None else min(ws_bytes, nb)
    _check(lib().dqrm_segment_sum_multi(tables.ref, batch, len(batches), arr, ws_bytes or 0, _stream(stream)),
           "dqrm_segment_sum_multi")


def dqrm_grad_quant_int8_multi(num_tables: int, dim: int, blocks, stream=None) -> None:
    """``blocks``: sequence of tuples (values, table_uniq_offsets, g_absmax, gq, g_scale) of device tensors, one per
    block (at most MAX_DEDUPE_BATCHES); the capacity of a block is the smaller first dimension of values and gq."""
    arr = (dqrm_quant_block_t * len(blocks))()
    for i, (v, tuo, am, gq, gs) in enumerate(blocks):
        arr[i] = dqrm_quant_block_t(min(v.shape[0], gq.shape[0]), _ptr(v), _ptr(tuo), _ptr(am), _ptr(gq), _ptr(gs))
    _check(lib().dqrm_grad_quant_int8_multi(num_tables, dim, len(blocks), arr, _stream(stream)),
           "dqrm_grad_quant_int8_multi")


def dqrm_grad_quant_int8(num_tables: int, dim: int, capacity: int, values: torch.Tensor,
                         table_uniq_offsets: torch.Tensor, g_absmax: torch.Tensor, gq: torch.Tensor,
                         g_scale: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_grad_quant_int8(num_tables, dim, capacity, _ptr(values), _ptr(table_uniq_offsets),
                                      _ptr(g_absmax), _ptr(gq), _ptr(g_scale), _stream(stream)),
           "dqrm_grad_quant_int8")


def dqrm_sparse_merge_workspace_bytes(num_tables: int, dim: int, num_blocks: int, max_total: int) -> int:
    return int(lib().dqrm_sparse_merge_workspace_bytes(num_tables, dim, num_blocks, max_total))


def dqrm_sparse_merge(tables: Tables, blocks, uniq_rows: torch.Tensor, table_uniq_offsets: torch.Tensor,
                      num_unique: torch.Tensor, sums: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """``blocks``: sequence of tuples (uniq_rows, table_uniq_offsets, gq) of device tensors, one per micro-batch
    (at most MAX_DEDUPE_BATCHES).  The outputs' first dimension is the capacity ``max_total``."""
    arr = (dqrm_sparse_block_t * len(blocks))()
    for i, (ur, tuo, gq) in enumerate(blocks):
        arr[i] = dqrm_sparse_block_t(_ptr(ur), _ptr(tuo), _ptr(gq), min(ur.shape[0], gq.shape[0]))
    _check(lib().dqrm_sparse_merge(tables.ref, len(blocks), arr, min(uniq_rows.shape[0], sums.shape[0]), _ptr(uniq_rows),
                                   _ptr(table_uniq_offsets), _ptr(num_unique), _ptr(sums), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)), "dqrm_sparse_merge")


def dqrm_sparse_update_sums(tables: Tables, capacity: int, uniq_rows: torch.Tensor, table_uniq_offsets: torch.Tensor,
                            sums: torch.Tensor, g_scale: torch.Tensor, lr: float, stream=None) -> None:
    _check(lib().dqrm_sparse_update_sums(tables.ref, capacity, _ptr(uniq_rows), _ptr(table_uniq_offsets), _ptr(sums),
                                         _ptr(g_scale), lr, _stream(stream)), "dqrm_sparse_update_sums")


def dqrm_sparse_update(tables: Tables, capacity: int, uniq_rows: torch.Tensor, table_uniq_offsets: torch.Tensor,
                       gq: torch.Tensor, g_scale: torch.Tensor, lr: float, stream=None) -> None:
    _check(lib().dqrm_sparse_update(tables.ref, capacity, _ptr(uniq_rows), _ptr(table_uniq_offsets), _ptr(gq),
                                    _ptr(g_scale), lr, _stream(stream)), "dqrm_sparse_update")


def dqrm_quant_update(tables: Tables, capacity: int, num_indices: int, values: torch.Tensor, uniq_rows: torch.Tensor,
                      table_uniq_offsets: torch.Tensor, g_absmax: torch.Tensor, gq: torch.Tensor,
                      g_scale: torch.Tensor, lr: float, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_quant_update(tables.ref, capacity, num_indices, _ptr(values), _ptr(uniq_rows),
                                   _ptr(table_uniq_offsets), _ptr(g_absmax), _ptr(gq), _ptr(g_scale), lr,
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "dqrm_quant_update")


class DenseModel:
    """Device copies of the MLP parameters and the C descriptor of the dense part of the model."""

    def __init__(self, num_tables: int, dim: int, bot_dims, bot_w, bot_b, top_dims, top_w, top_b, device):
        to_dev = lambda lst: [torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(device) for a in lst]
        self.bot_w, self.bot_b, self.top_w, self.top_b = to_dev(bot_w), to_dev(bot_b), to_dev(top_w), to_dev(top_b)
        self.bot_dims = np.ascontiguousarray(bot_dims, np.int32)
        self.top_dims = np.ascontiguousarray(top_dims, np.int32)
        ptrs = lambda lst: (C.c_void_p * len(lst))(*[t.data_ptr() for t in lst])
        self._pw = [ptrs(self.bot_w), ptrs(self.bot_b), ptrs(self.top_w), ptrs(self.top_b)]
        addr = lambda a: C.cast(a, C.c_void_p).value
        self.c = dqrm_dense_model_t(int(self.bot_dims[0]), num_tables, dim, len(self.bot_w),
                                    self.bot_dims.ctypes.data, addr(self._pw[0]), addr(self._pw[1]),
                                    len(self.top_w), self.top_dims.ctypes.data, addr(self._pw[2]), addr(self._pw[3]))
        self.num_tables, self.dim = num_tables, dim

    @property
    def ref(self):
        return C.byref(self.c)


def dqrm_dense_workspace_bytes(model: DenseModel, batch: int) -> int:
    return int(lib().dqrm_dense_workspace_bytes(model.ref, batch))


def dqrm_dense_step(model: DenseModel, batch: int, dense_x: torch.Tensor, emb_out: torch.Tensor,
                    labels: torch.Tensor, lr: float, loss: torch.Tensor, grad_emb: torch.Tensor,
                    workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_dense_step(model.ref, batch, _ptr(dense_x), _ptr(emb_out), _ptr(labels), lr, _ptr(loss),
                                 _ptr(grad_emb), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                 _stream(stream)), "dqrm_dense_step")


def dqrm_dense_param_count(model: DenseModel) -> int:
    return int(lib().dqrm_dense_param_count(model.ref))


class DenseQuant:
    """Descriptor of the quantised variants of the dense step; the tensors (device) stay owned by the caller."""

    def __init__(self, weight_bits: int = 0, grad_bits: int = 0, grad_error: Optional[torch.Tensor] = None,
                 grad_scale: Optional[torch.Tensor] = None, grad_codes: Optional[torch.Tensor] = None,
                 grads: Optional[torch.Tensor] = None, wq: Optional[torch.Tensor] = None,
                 grad_buffer: Optional[torch.Tensor] = None, buffer_add: bool = False, buffer_update: bool = False):
        self._keep = (grad_error, grad_scale, grad_codes, grads, wq, grad_buffer)
        p = lambda t: t.data_ptr() if t is not None else None
        self.c = dqrm_dense_quant_t(weight_bits, grad_bits, p(grad_error), p(grad_scale), p(grad_codes), p(grads), p(wq),
                                    p(grad_buffer), int(buffer_add), int(buffer_update))

    @property
    def ref(self):
        return C.byref(self.c)


def dqrm_dense_step_quant(model: DenseModel, quant: Optional[DenseQuant], batch: int, dense_x: torch.Tensor,
                          emb_out: torch.Tensor, labels: torch.Tensor, lr: float, loss: torch.Tensor,
                          grad_emb: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().dqrm_dense_step_quant(model.ref, quant.ref if quant is not None else None, batch, _ptr(dense_x),
                                       _ptr(emb_out), _ptr(labels), lr, _ptr(loss), _ptr(grad_emb), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)),
           "dqrm_dense_step_quant")


def dqrm_check_status(stream=None) -> Tuple[int, int, int]:
    """(code, table, value); code 0 = no data-dependent problem since the last call.  Synchronises."""
    t, v = C.c_int32(-1), C.c_int64(-1)
    rc = lib().dqrm_check_status(_stream(stream), C.byref(t), C.byref(v))
    if rc == ERR_HIP:
        _check(rc, "dqrm_check_status")
    return int(rc), int(t.value), int(v.value)


class StepBuffers:
    """Device buffers one training step needs, allocated once (the library itself allocates nothing)."""

    def __init__(self, T: int, D: int, B: int, N: int, device, want_codes: bool = False):
        cap = max(N, 1)
        i32, i64, f32 = torch.int32, torch.int64, torch.float32
        self.T, self.D, self.B, self.N, self.cap = T, D, B, N, cap
        self.out = torch.empty((B, T, D), dtype=f32, device=device)
        self.codes = torch.empty((cap, D), dtype=torch.int8, device=device) if want_codes else None
        self.sorted_pos = torch.empty(cap, dtype=i32, device=device)
        self.uniq_rows = torch.empty(cap, dtype=i64, device=device)
        self.seg_offsets = torch.empty(cap + 1, dtype=i32, device=device)
        self.table_uniq_offsets = torch.empty(T + 1, dtype=i32, device=device)
        self.num_unique = torch.empty(1, dtype=i32, device=device)
        self.values = torch.empty((cap, D), dtype=f32, device=device)
        self.g_absmax = torch.empty(T, dtype=f32, device=device)
        self.gq = torch.empty((cap, D), dtype=torch.int8, device=device)
        self.g_scale = torch.empty(T, dtype=f32, device=device)
        nbytes = dqrm_embbag_bwd_workspace_bytes(T, D, B, N)
        if nbytes == 0:
            raise DqrmError(ERR_UNSUPPORTED, "dqrm_embbag_bwd_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)


def dqrm_fwd_bwd_step(tables: Tables, bufs: StepBuffers, indices: torch.Tensor, offsets: torch.Tensor,
                      grad_out: torch.Tensor, lr: float, mode: int = FWD_MASTER, stream=None) -> None:
    """One pass of the whole hot path on one stream, no host sync: forward, dedupe, segment sums, INT8 codes and update.

    What dqrm_embbag_fwd, dqrm_dedupe, dqrm_segment_sum and dqrm_quant_update leave in ``bufs`` and the tables, bit for bit, in fewer
    launches where the batch allows it."""
    b = bufs
    _check(lib().dqrm_fwd_bwd_step(tables.ref, _ptr(indices), _ptr(offsets), b.B, indices.numel(), mode, _ptr(b.out), _ptr(b.codes),
                                   _ptr(grad_out), lr, b.cap, _ptr(b.sorted_pos), _ptr(b.uniq_rows), _ptr(b.seg_offsets),
                                   _ptr(b.table_uniq_offsets), _ptr(b.num_unique), _ptr(b.values), _ptr(b.g_absmax), _ptr(b.gq),
                                   _ptr(b.g_scale), _ptr(b.workspace), b.workspace.numel() * b.workspace.element_size(),
                                   _stream(stream)), "dqrm_fwd_bwd_step")


# ---- layer norm and MXFP4 linear layers ---------------------------------------------------------------------------------


# Operands have to be in the memory of one GPU, that of a call's first matrix: the library cannot see where they are.
# (These run on every call, and a call on little data is as long as they are: no loops, no formatting unless something is wrong.)
def _matrix(t: torch.Tensor, what: str) -> Tuple[int, int, int, int, int, int]:
    """(element type, rows, columns, address, row stride, GPU) of a matrix whose rows' elements lie one behind the other."""
    dtype, shape = _DTYPES.get(t.dtype), t.shape
    if dtype is None or len(shape) != 2:
        raise AssertionError(f"{what}: a matrix of float32, bfloat16 or float16")
    rows, cols = shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise AssertionError(f"{what}: the elements of a row must be contiguous")
    return dtype, rows, cols, t.data_ptr(), ld, t.get_device()


def _rows_of(t: torch.Tensor, rows: int, cols: int, dtype, what: str, gpu: int) -> Tuple[int, int]:
    """(address, row stride) of another one of this kind."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 2 or shape[0] != rows or shape[1] != cols:
        raise AssertionError(f"{what}: ({rows}, {cols}) of {dtype}, got {tuple(shape)} of {t.dtype}")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise AssertionError(f"{what}: the elements of a row must be contiguous")
    if t.get_device() != gpu:
        raise _elsewhere(what)
    return t.data_ptr(), ld


def _vector(t: Optional[torch.Tensor], n: int, what: str, gpu: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise AssertionError(f"{what}: {n} contiguous float32 values")
    if t.get_device() != gpu:
        raise _elsewhere(what)
    return t.data_ptr()


def _space(ws: Optional[torch.Tensor], gpu: int) -> Tuple[Optional[int], int]:
    if ws is None:
        return None, 0
    if not ws.is_contiguous():
        raise AssertionError("workspace: contiguous memory")
    if ws.get_device() != gpu:
        raise _elsewhere("workspace")
    return ws.data_ptr(), ws.nbytes


def _elsewhere(what: str) -> DqrmError:
    return DqrmError(ERR_INVALID_ARG, what, "not in the memory that the other operands are in")


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _there(gpu: int, call, *args) -> None:
    """The call again with the operands' GPU the current one: a default stream's handle is null for every GPU."""
    with torch.cuda.device(gpu):
        call(*args)


def _stream_of(gpu: int, stream) -> Optional[int]:
    """The stream asked for, or the current one of the GPU that the operands are on."""
    if gpu < 0:
        raise DqrmError(ERR_INVALID_ARG, "operands", "in host memory")
    if stream is None and _raw_stream is not None:
        return _raw_stream(gpu)
    return _stream(stream)


class MxMatrix:
    """A matrix in MXFP4 (see ``dqrm_mxfp4_t``): the device buffers of its codes and scales and the C descriptor.  Buffers that are not
    given are made on ``device``: by default where the given one is, or else on torch's default device, or, that being the host, on the
    current GPU (host memory where there is none: no call takes such a matrix)."""

    def __init__(self, rows: int, cols: int, device=None, codes: Optional[torch.Tensor] = None,
                 scales: Optional[torch.Tensor] = None):
        self.rows, self.cols = int(rows), int(cols)
        groups = -(-self.cols // 128)
        if device is None and (codes is None or scales is None):
            given = codes if codes is not None else scales
            device = given.device if given is not None else torch.get_default_device()
            if given is None and device.type == "cpu" and torch.cuda.is_available():
                device = "cuda"
        byte = lambda n: torch.empty((self.rows, n), dtype=torch.uint8, device=device)  # noqa: E731
        self.codes = codes if codes is not None else byte(64 * groups)
        self.scales = scales if scales is not None else byte(4 * groups)
        self.gpu = self.codes.get_device()  # -1: host memory
        for t, n in ((self.codes, 64 * groups), (self.scales, 4 * groups)):
            _rows_of(t, self.rows, n, torch.uint8, "MxMatrix", self.gpu)
        self.c = dqrm_mxfp4_t(self.rows, self.cols, _ptr(self.codes), _ptr(self.scales))
        self.ref = C.byref(self.c)


def _mx(q: Optional[MxMatrix], what: str, gpu: int):
    if q is None:
        return None
    if q.gpu != gpu:
        raise _elsewhere(what)
    return q.ref


def dqrm_mxfp4_quant_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().dqrm_mxfp4_quant_workspace_bytes(rows, cols))


def dqrm_mxfp4_quant(x: torch.Tensor, by_rows: Optional[MxMatrix] = None, by_cols: Optional[MxMatrix] = None,
                     gate: Optional[torch.Tensor] = None, col_sums: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    dtype, R, D, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_mxfp4_quant, x, by_rows, by_cols, gate, col_sums, workspace, stream)
    pg, ldg = (None, 0) if gate is None else _rows_of(gate, R, D, x.dtype, "gate", gpu)
    rc = lib().dqrm_mxfp4_quant(
        dtype, R, D, p, ld, pg, ldg, _mx(by_rows, "by_rows", gpu), _mx(by_cols, "by_cols", gpu),
        _vector(col_sums, D, "col_sums", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_mxfp4_quant")


def dqrm_mxfp4_dequant(q: MxMatrix, out: torch.Tensor, stream=None) -> None:
    dtype, R, D, p, ld, gpu = _matrix(out, "out")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_mxfp4_dequant, q, out, stream)
    if R != q.rows or D != q.cols:
        raise AssertionError(f"out: ({q.rows}, {q.cols}), got ({R}, {D})")
    rc = lib().dqrm_mxfp4_dequant(
        _mx(q, "q", gpu), dtype, p, ld, _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_mxfp4_dequant")


def dqrm_mxfp4_matmul_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(lib().dqrm_mxfp4_matmul_workspace_bytes(m, n, k))


def dqrm_mxfp4_matmul(a: MxMatrix, b: MxMatrix, out: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    dtype, m, n, po, ldo, gpu = _matrix(out, "out")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_mxfp4_matmul, a, b, out, bias, relu, workspace, stream)
    if m != a.rows or n != b.rows:
        raise AssertionError(f"out: ({a.rows}, {b.rows}), got ({m}, {n})")
    rc = lib().dqrm_mxfp4_matmul(
        _mx(a, "a", gpu), _mx(b, "b", gpu), _vector(bias, n, "bias", gpu), relu, dtype, po, ldo,
        *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_mxfp4_matmul")


def dqrm_mxfp4_linear_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(lib().dqrm_mxfp4_linear_workspace_bytes(m, n, k))


def dqrm_mxfp4_linear(x: torch.Tensor, w: MxMatrix, out: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False,
                      gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, eps: Optional[float] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """``eps`` given: x goes through a layer norm (with ``gamma`` and ``beta`` if given) first."""
    dtype, m, k, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_mxfp4_linear, x, w, out, bias, relu, gamma, beta, eps, workspace, stream)
    if k != w.cols:
        raise AssertionError(f"x: ({m}, {w.cols}), got ({m}, {k})")
    po, ldo = _rows_of(out, m, w.rows, x.dtype, "out", gpu)
    rc = lib().dqrm_mxfp4_linear(
        dtype, m, p, ld, eps is not None, _vector(gamma, k, "gamma", gpu), _vector(beta, k, "beta", gpu),
        eps or 0.0, _mx(w, "w", gpu), _vector(bias, w.rows, "bias", gpu), relu, po, ldo, *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_mxfp4_linear")


def dqrm_layernorm_fwd(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float,
                       y: Optional[torch.Tensor] = None, mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                       q: Optional[MxMatrix] = None, stream=None) -> None:
    dtype, R, D, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_layernorm_fwd, x, gamma, beta, eps, y, mean, rstd, q, stream)
    py, ldy = (None, 0) if y is None else _rows_of(y, R, D, x.dtype, "y", gpu)
    rc = lib().dqrm_layernorm_fwd(
        dtype, R, D, p, ld, _vector(gamma, D, "gamma", gpu), _vector(beta, D, "beta", gpu), eps, py, ldy,
        _vector(mean, R, "mean", gpu), _vector(rstd, R, "rstd", gpu), _mx(q, "q", gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_layernorm_fwd")


def dqrm_layernorm_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().dqrm_layernorm_bwd_workspace_bytes(rows, cols))


def dqrm_layernorm_bwd(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, gamma: Optional[torch.Tensor],
                       dx: Optional[torch.Tensor] = None, dgamma: Optional[torch.Tensor] = None,
                       dbeta: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    dtype, R, D, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_layernorm_bwd, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, workspace, stream)
    pdy, lddy = _rows_of(dy, R, D, x.dtype, "dy", gpu)
    pdx, lddx = (None, 0) if dx is None else _rows_of(dx, R, D, x.dtype, "dx", gpu)
    rc = lib().dqrm_layernorm_bwd(
        dtype, R, D, pdy, lddy, p, ld, _vector(mean, R, "mean", gpu), _vector(rstd, R, "rstd", gpu),
        _vector(gamma, D, "gamma", gpu), pdx, lddx, _vector(dgamma, D, "dgamma", gpu), _vector(dbeta, D, "dbeta", gpu),
        *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_layernorm_bwd")


# ---- residual norms, a loss over many classes, the clip of all gradients -----------------------------------------------------


class ResidualNorm:
    """Descriptor of the norms around a residual join (see ``dqrm_residual_norm_t``); the vectors (device, float32) stay owned by the
    caller.  They have to be contiguous, of one length and in one GPU's memory."""

    def __init__(self, post: int = NORM_NONE, pre: int = NORM_RMS, post_gamma: Optional[torch.Tensor] = None, post_beta: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, pre_gamma: Optional[torch.Tensor] = None, pre_beta: Optional[torch.Tensor] = None,
                 res_scale: float = 1.0, post_eps: float = 1e-5, pre_eps: float = 1e-5):
        vectors = (post_gamma, post_beta, gate, pre_gamma, pre_beta)
        given = [v for v in vectors if v is not None]
        self.cols = given[0].numel() if given else None  # None: any
        self.gpu = given[0].get_device() if given else None
        self._keep = vectors
        p = [_vector(v, self.cols, "ResidualNorm", self.gpu) for v in vectors]
        self.c = dqrm_residual_norm_t(post, pre, *p, res_scale, post_eps, pre_eps)
        self.ref = C.byref(self.c)


def _norm_of(norm: ResidualNorm, cols: int, gpu: int):
    if norm.cols is not None and norm.cols != cols:
        raise AssertionError(f"norm: vectors of {cols}, got {norm.cols}")
    if norm.gpu is not None and norm.gpu != gpu:
        raise _elsewhere("norm")
    return norm.ref


def _rows_block(t: Optional[torch.Tensor], n: int, cols: int, what: str, gpu: int) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (n, cols) or not t.is_contiguous():
        raise AssertionError(f"{what}: ({n}, {cols}) contiguous float32 values")
    if t.get_device() != gpu:
        raise _elsewhere(what)
    return t.data_ptr()


def dqrm_residual_norm_fwd(norm: ResidualNorm, u: torch.Tensor, r: torch.Tensor, out: torch.Tensor, y: Optional[torch.Tensor] = None,
                           stats: Optional[torch.Tensor] = None, q: Optional[MxMatrix] = None, stream=None) -> None:
    dtype, R, D, p, ld, gpu = _matrix(u, "u")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_residual_norm_fwd, norm, u, r, out, y, stats, q, stream)
    pr, ldr = _rows_of(r, R, D, u.dtype, "r", gpu)
    po, ldo = _rows_of(out, R, D, u.dtype, "out", gpu)
    py, ldy = (None, 0) if y is None else _rows_of(y, R, D, u.dtype, "y", gpu)
    rc = lib().dqrm_residual_norm_fwd(
        dtype, R, D, _norm_of(norm, D, gpu), p, ld, pr, ldr, po, ldo, py, ldy, _rows_block(stats, 4, R, "stats", gpu), _mx(q, "q", gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_residual_norm_fwd")


def dqrm_residual_norm_bwd_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().dqrm_residual_norm_bwd_workspace_bytes(rows, cols))


def dqrm_residual_norm_bwd(norm: ResidualNorm, dout: Optional[torch.Tensor], dy: Optional[torch.Tensor], u: Optional[torch.Tensor],
                           out: Optional[torch.Tensor], stats: Optional[torch.Tensor], du: Optional[torch.Tensor] = None,
                           dr: Optional[torch.Tensor] = None, dparams: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           stream=None) -> None:
    """``u`` may be None without a norm behind the block and without ``dparams``, ``dy`` and ``out`` without one before the next."""
    first = dout if dout is not None else dy
    if first is None:
        raise AssertionError("dout or dy: a gradient")
    dtype, R, D, _, _, gpu = _matrix(first, "dout" if dout is not None else "dy")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_residual_norm_bwd, norm, dout, dy, u, out, stats, du, dr, dparams, workspace, stream)
    at = lambda t, what: (None, 0) if t is None else _rows_of(t, R, D, first.dtype, what, gpu)  # noqa: E731
    rc = lib().dqrm_residual_norm_bwd(
        dtype, R, D, _norm_of(norm, D, gpu), *at(dout, "dout"), *at(dy, "dy"), *at(u, "u"), *at(out, "out"), _rows_block(stats, 4, R, "stats", gpu),
        *at(du, "du"), *at(dr, "dr"), _rows_block(dparams, 5, D, "dparams", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_residual_norm_bwd")


def _targets_of(t: torch.Tensor, rows: int, gpu: int) -> int:
    if t.dtype is not torch.int64 or t.shape != (rows,) or not t.is_contiguous():
        raise AssertionError(f"targets: {rows} contiguous int64 values")
    if t.get_device() != gpu:
        raise _elsewhere("targets")
    return t.data_ptr()


def dqrm_softmax_xent_fwd_workspace_bytes(rows: int, classes: int, width: int, dtype: torch.dtype) -> int:
    return int(lib().dqrm_softmax_xent_fwd_workspace_bytes(rows, classes, width, _DTYPES[dtype]))


def dqrm_softmax_xent_fwd(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, loss: torch.Tensor, lse: torch.Tensor,
                          bias: Optional[torch.Tensor] = None, scale: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    dtype, M, K, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_softmax_xent_fwd, x, w, targets, loss, lse, bias, scale, workspace, stream)
    V = w.shape[0]
    pw, ldw = _rows_of(w, V, K, x.dtype, "w", gpu)
    rc = lib().dqrm_softmax_xent_fwd(
        dtype, M, V, K, p, ld, pw, ldw, _vector(bias, V, "bias", gpu), scale, _targets_of(targets, M, gpu), _vector(loss, M, "loss", gpu),
        _vector(lse, M, "lse", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_softmax_xent_fwd")


def dqrm_softmax_xent_bwd_workspace_bytes(rows: int, classes: int, width: int, dtype: torch.dtype) -> int:
    return int(lib().dqrm_softmax_xent_bwd_workspace_bytes(rows, classes, width, _DTYPES[dtype]))


def dqrm_softmax_xent_bwd(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, grad: torch.Tensor,
                          dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                          bias: Optional[torch.Tensor] = None, scale: float = 1.0, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """``lse``: the forward's; ``grad``: the gradients of the rows' losses (1 / rows each for their mean)."""
    dtype, M, K, p, ld, gpu = _matrix(x, "x")
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_softmax_xent_bwd, x, w, targets, lse, grad, dx, dw, dbias, bias, scale, workspace, stream)
    V = w.shape[0]
    pw, ldw = _rows_of(w, V, K, x.dtype, "w", gpu)
    pdx, lddx = (None, 0) if dx is None else _rows_of(dx, M, K, x.dtype, "dx", gpu)
    pdw, lddw = (None, 0) if dw is None else _rows_of(dw, V, K, x.dtype, "dw", gpu)
    rc = lib().dqrm_softmax_xent_bwd(
        dtype, M, V, K, p, ld, pw, ldw, _vector(bias, V, "bias", gpu), scale, _targets_of(targets, M, gpu), _vector(lse, M, "lse", gpu),
        _vector(grad, M, "grad", gpu), pdx, lddx, pdw, lddw, _vector(dbias, V, "dbias", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_softmax_xent_bwd")


def _grad_rows(t: torch.Tensor) -> Tuple[int, int, int]:
    """(rows, columns, row stride): a tensor whose values lie one behind the other is one row, but a matrix keeps its rows."""
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] <= 1):
        return t.shape[0], t.shape[1], t.stride(0)
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    if t.dim() == 1:  # a column
        return t.shape[0], 1, t.stride(0)
    raise AssertionError("a gradient: contiguous, or a matrix whose rows are")


class Grads:
    """Gradient tensors of any shapes, float32, bfloat16 and float16 mixed, in one GPU's memory, and the C descriptors (see ``dqrm_grad_t``):
    made once for the buffers that a program keeps its gradients in, which stay owned by the caller.  ``out``: as many tensors of the same
    shapes and types, or None: scaled in place.  ``counts``: {number of a tensor (a matrix): int32 tensor of one value, how many of its rows
    are there}."""

    def __init__(self, tensors, out=None, counts=None):
        tensors = list(tensors)
        outs = [None] * len(tensors) if out is None else list(out)
        counts = dict(counts or {})
        if len(outs) != len(tensors) or not all(0 <= k < len(tensors) for k in counts):
            raise AssertionError("Grads: an output to each tensor, counts of tensors that are there")
        self._keep = (tensors, outs, counts)
        self.n = len(tensors)
        self.gpu = tensors[0].get_device() if tensors else None
        self.c = (dqrm_grad_t * max(self.n, 1))()
        for k, (t, o) in enumerate(zip(tensors, outs)):
            dtype = _DTYPES.get(t.dtype)
            if dtype is None or (o is not None and (o.dtype is not t.dtype or o.shape != t.shape)):
                raise AssertionError("Grads: float32, bfloat16 or float16, and outputs of the same shapes and types")
            count = counts.get(k)
            if count is not None and (count.dtype is not torch.int32 or count.numel() != 1 or t.dim() != 2):
                raise AssertionError("Grads: a count is one int32 value, of a matrix")
            if any(v is not None and v.get_device() != self.gpu for v in (t, o, count)):
                raise _elsewhere("Grads")
            rows, cols, ld = _grad_rows(t)
            ld_out = 0
            if o is not None:
                same = _grad_rows(o)
                if same[:2] != (rows, cols):
                    raise AssertionError("Grads: an output laid out like its tensor")
                ld_out = same[2]
            self.c[k] = dqrm_grad_t(t.data_ptr(), rows, cols, ld, None if o is None else o.data_ptr(), ld_out, None if count is None else count.data_ptr(), dtype)


def dqrm_grad_workspace_bytes(grads: Grads) -> int:
    return int(lib().dqrm_grad_workspace_bytes(grads.c, grads.n))


def _scalar(t: torch.Tensor, what: str, gpu: Optional[int]) -> Tuple[int, int]:
    """(address, GPU) of one float32 value"""
    if t.dtype is not torch.float32 or t.numel() != 1:
        raise AssertionError(f"{what}: one float32 value")
    if gpu is not None and t.get_device() != gpu:
        raise _elsewhere(what)
    return t.data_ptr(), t.get_device()


def dqrm_grad_norm(grads: Grads, norm: torch.Tensor, kind: int = GRAD_NORM_2, norms: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    p, gpu = _scalar(norm, "norm", grads.gpu)
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_grad_norm, grads, norm, kind, norms, workspace, stream)
    rc = lib().dqrm_grad_norm(grads.c, grads.n, kind, p, _vector(norms, grads.n, "norms", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_grad_norm")


def dqrm_grad_scale(grads: Grads, norm: torch.Tensor, max_norm: float, stream=None) -> None:
    p, gpu = _scalar(norm, "norm", grads.gpu)
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_grad_scale, grads, norm, max_norm, stream)
    rc = lib().dqrm_grad_scale(grads.c, grads.n, p, max_norm, _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_grad_scale")


def dqrm_grad_clip(grads: Grads, max_norm: float, norm: torch.Tensor, kind: int = GRAD_NORM_2, norms: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    p, gpu = _scalar(norm, "norm", grads.gpu)
    if gpu >= 0 and gpu != _current_device():
        return _there(gpu, dqrm_grad_clip, grads, max_norm, norm, kind, norms, workspace, stream)
    rc = lib().dqrm_grad_clip(grads.c, grads.n, kind, max_norm, p, _vector(norms, grads.n, "norms", gpu), *_space(workspace, gpu), _stream_of(gpu, stream))
    if rc != OK:
        _check(rc, "dqrm_grad_clip")
