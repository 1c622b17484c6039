"""ctypes binding of libmarcache.so (argument marshalling only).

Every function here forwards to the C ABI declared in include/mar_cache.h,
include/mar_kernels.h and include/mar_head.h; every step of the computation runs in the HIP
library.  PyTorch supplies device memory and the current stream.  There is
no fallback: if the library is missing or fails to load, an ImportError /
OSError is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmarcache.so")

MAR_OK, MAR_E_ARG, MAR_E_SHAPE, MAR_E_STATE, MAR_E_WORKSPACE, MAR_E_DEVICE, MAR_E_HOST = 0, -1, -2, -3, -4, -5, -6
MAR_F32, MAR_BF16 = 0, 1
MAR_FULL, MAR_TOKEN_CACHED, MAR_TOKEN_GIVEN, MAR_TOKEN_CACHED_MOST_SIMILAR = 0, 1, 2, 3
MAR_CFG_STORE, MAR_CFG_REUSE = 0, 1
MAR_SCORE_VALUES, MAR_SCORE_FEATURES = 0, 1
MAR_ROTARY_HALVES, MAR_ROTARY_NEIGHBOURS = 0, 1
PROF_KINDS = ("qkv", "proj", "fc1", "fc2", "attention", "layernorm", "scores", "select", "cfg")

STATUS_NAMES = {0: "MAR_OK", -1: "MAR_E_ARG", -2: "MAR_E_SHAPE", -3: "MAR_E_STATE",
                -4: "MAR_E_WORKSPACE", -5: "MAR_E_DEVICE", -6: "MAR_E_HOST"}

# every symbol the headers declare (checked by the CPU tests)
EXPORTED = (
    "mar_workspace_bytes", "mar_cache_init", "mar_step", "mar_cfg_combine", "mar_output",
    "mar_cache_destroy", "mar_last_error", "mar_profile_start", "mar_profile_stop",
    "mar_k_layernorm", "mar_k_linear", "mar_k_linear_residual", "mar_k_qkv",
    "mar_k_attention", "mar_k_scores", "mar_k_select", "mar_k_select_most_similar",
    "mar_k_gemm_variant",
    "mar_k_rotary", "mar_k_paged_store", "mar_k_paged_attention", "mar_k_paged_attention_workspace_bytes",
    "mar_k_paged_tree_attention", "mar_k_paged_tree_attention_workspace_bytes", "mar_k_probabilities",
    "mar_k_draft_verify", "mar_k_draft_verify_workspace_bytes", "mar_k_paged_keep", "mar_k_paged_fork",
    "mar_k_paged_fork_workspace_bytes",
    "mar_head_workspace_bytes", "mar_head_init", "mar_head_sample", "mar_head_destroy",
    "mar_head_sample_noalloc",
)
GEMM_VARIANTS = 16


class MarError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class MarDimsC(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("d_mlp", ctypes.c_int32),
                ("seq_len", ctypes.c_int32), ("max_slots", ctypes.c_int32),
                ("full_prefix", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("ln_eps", ctypes.c_float), ("score_source", ctypes.c_int32),
                ("fresh_kv", ctypes.c_int32)]


WEIGHT_FIELDS = ("ln1_w", "ln1_b", "qkv_w", "qkv_b", "proj_w", "proj_b",
                 "ln2_w", "ln2_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b")


class MarBlockWeightsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in WEIGHT_FIELDS]


class MarHeadDimsC(ctypes.Structure):
    _fields_ = [("width", ctypes.c_int32), ("depth", ctypes.c_int32), ("cond_dim", ctypes.c_int32),
                ("token_dim", ctypes.c_int32), ("steps", ctypes.c_int32), ("train_steps", ctypes.c_int32),
                ("freq_dim", ctypes.c_int32), ("max_rows", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("beta_start", ctypes.c_float), ("beta_end", ctypes.c_float), ("ln_eps", ctypes.c_float)]


HEAD_WEIGHT_FIELDS = ("z_w", "z_b", "t1_w", "t1_b", "t2_w", "t2_b", "in_w", "in_b", "ada_w", "ada_b",
                      "fc1_w", "fc1_b", "fc2_w", "fc2_b", "out_w", "out_b")


class MarHeadWeightsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in HEAD_WEIGHT_FIELDS]


class MarRotaryC(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("n_pairs", ctypes.c_int32),
                ("n_axes", ctypes.c_int32), ("layout", ctypes.c_int32)]


class MarPagedBatchC(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "table", "q_start", "kv_len")] +
                [(n, ctypes.c_int32) for n in ("n_pages", "n_heads", "page", "d_head", "n_seqs", "max_pages",
                                               "max_kv")])


_vp, _i32, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
_i64 = ctypes.c_int64
_SIGNATURES = {
    "mar_workspace_bytes": (_sz, [ctypes.POINTER(MarDimsC)]),
    "mar_cache_init": (_i32, [ctypes.POINTER(MarDimsC), ctypes.POINTER(MarBlockWeightsC), _vp, _sz, _vp,
                              ctypes.POINTER(_vp)]),
    "mar_step": (_i32, [_vp, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _vp]),
    "mar_cfg_combine": (_i32, [_vp, _vp, _vp, _i32, _i32, _i32, _f32, _vp, _vp, _vp]),
    "mar_output": (_vp, [_vp]),
    "mar_cache_destroy": (_i32, [_vp]),
    "mar_last_error": (ctypes.c_char_p, []),
    "mar_profile_start": (_i32, [_vp, _i32]),
    "mar_profile_stop": (_i32, [_vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64),
                                ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
    "mar_k_layernorm": (_i32, [_i32, _vp, _i32, _vp, _i32, _i32, _i32, _i32, _vp, _vp, _f32, _vp, _vp, _vp]),
    "mar_k_linear": (_i32, [_i32, _i32, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp]),
    "mar_k_linear_residual": (_i32, [_i32, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _i32, _i32,
                                     _vp, _vp]),
    "mar_k_qkv": (_i32, [_i32, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp,
                         _vp, _vp, _vp]),
    "mar_k_attention": (_i32, [_i32, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _i32, _i32, _vp]),
    "mar_k_scores": (_i32, [_i32, _vp, _vp, _i32, _i32, _i32, _i32, _vp, _i32, _vp]),
    "mar_k_select": (_i32, [_vp, _i32, _i32, _i32, _vp, _vp]),
    "mar_k_select_most_similar": (_i32, [_vp, _i32, _i32, _i32, _vp, _vp]),
    "mar_k_gemm_variant": (_i32, [_i32]),
    "mar_k_rotary": (_i32, [_i32, ctypes.POINTER(MarRotaryC), _vp, _i64, _vp, _i32, _i32, _i32, _vp, _i64, _vp]),
    "mar_k_paged_store": (_i32, [_i32, ctypes.POINTER(MarPagedBatchC), ctypes.POINTER(MarRotaryC), _vp, _i32, _vp,
                                 _i64, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp]),
    "mar_k_paged_attention": (_i32, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _i32, _vp, _i64, _i32, _i32, _i32,
                                     _vp, _sz, _vp, _i64, _vp]),
    "mar_k_paged_attention_workspace_bytes": (_sz, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _i32, _i32, _i32]),
    "mar_k_paged_tree_attention": (_i32, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _i32, _vp, _i64, _vp, _i32, _i32,
                                          _vp, _sz, _vp, _i64, _vp]),
    "mar_k_paged_tree_attention_workspace_bytes": (_sz, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _i32, _i32,
                                                         _i32]),
    "mar_k_probabilities": (_i32, [_i32, _vp, _i64, _vp, _i32, _i32, _vp, _i64, _vp]),
    "mar_k_draft_verify": (_i32, [_i32, _i32, _vp, _i32, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _vp, _sz, _vp]),
    "mar_k_draft_verify_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "mar_k_paged_keep": (_i32, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _vp, _vp, _vp, _vp]),
    "mar_k_paged_fork": (_i32, [_i32, ctypes.POINTER(MarPagedBatchC), _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                _vp]),
    "mar_k_paged_fork_workspace_bytes": (_sz, [ctypes.POINTER(MarPagedBatchC), _i32]),
    "mar_head_workspace_bytes": (_sz, [ctypes.POINTER(MarHeadDimsC)]),
    "mar_head_init": (_i32, [ctypes.POINTER(MarHeadDimsC), ctypes.POINTER(MarHeadWeightsC), _vp, _sz, _vp,
                             ctypes.POINTER(_vp)]),
    "mar_head_sample": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _f32, _vp, _vp, _vp, _vp]),
    "mar_head_destroy": (_i32, [_vp]),
    "mar_head_sample_noalloc": (_i32, [_vp, _vp, _vp, _i32, _vp, _vp, _i32, _vp, _vp, _f32, _vp, _vp, _vp,
                                       _vp]),
}

_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built: run `python -m paper_2503_12450_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != MAR_OK:
        raise MarError(status, load().mar_last_error().decode())


def dtype_code(dtype: str) -> int:
    return {"f32": MAR_F32, "bf16": MAR_BF16}[dtype]


SCORE_SOURCES = {"values": MAR_SCORE_VALUES, "features": MAR_SCORE_FEATURES}


def dims_c(dims) -> MarDimsC:
    return MarDimsC(dims.n_layers, dims.d_model, dims.n_heads, dims.d_mlp, dims.seq_len,
                    dims.max_slots, dims.full_prefix, dtype_code(dims.dtype), dims.ln_eps,
                    SCORE_SOURCES[getattr(dims, "score_source", "values")],
                    1 if getattr(dims, "fresh_kv", False) else 0)


# --------------------------------------------------------------------------
# torch plumbing
# --------------------------------------------------------------------------

def _torch():
    import torch
    return torch


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    device = torch.cuda.current_device()
    # the current stream's handle without a Stream object around it (0.3 us
    # instead of 2.8, of a call that takes 4 to launch a small kernel)
    try:
        return torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:  # not a public name
        return torch.cuda.current_stream(device).cuda_stream


def workspace_bytes(dims) -> int:
    d = dims_c(dims)
    n = load().mar_workspace_bytes(ctypes.byref(d))
    if n == 0:
        raise MarError(MAR_E_SHAPE, load().mar_last_error().decode())
    return n


class MarCache:
    """Handle over a workspace tensor; the library copies the weights in."""

    def __init__(self, dims, blocks: Sequence[Dict[str, "object"]], device="cuda", stream=None):
        torch = _torch()
        self.dims = dims
        self.lib = load()
        nbytes = workspace_bytes(dims)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.workspace.data_ptr()) % 256
        self._ws = self.workspace[off:off + nbytes]
        arr = (MarBlockWeightsC * dims.n_layers)()
        for i, blk in enumerate(blocks):
            for f in WEIGHT_FIELDS:
                setattr(arr[i], f, blk[f].data_ptr())
        self._blocks = blocks  # kept alive until the copies are done
        handle = ctypes.c_void_p()
        d = dims_c(dims)
        _check(self.lib.mar_cache_init(ctypes.byref(d), arr, self._ws.data_ptr(), nbytes,
                                       _stream(stream), ctypes.byref(handle)))
        self.handle = handle

    def close(self) -> None:
        if getattr(self, "handle", None):
            self.lib.mar_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, x, mode: int, n_recompute: int = 0, slot0: int = 0, y=None, sel_idx=None,
             stream=None) -> None:
        n_slots = x.shape[0]
        if mode == MAR_TOKEN_GIVEN and sel_idx is not None:
            import numpy as np
            host = np.ascontiguousarray(sel_idx, dtype=np.int32)
            self._given = host  # stays alive while the upload is in flight
            idx_ptr = host.ctypes.data
        else:
            idx_ptr = _ptr(sel_idx)
        _check(self.lib.mar_step(self.handle, x.data_ptr(), _ptr(y), slot0, n_slots, mode,
                                 n_recompute, idx_ptr, _stream(stream)))

    def cfg_combine(self, op: int, y_cond, y_uncond, scale: float, guided, uncond_out=None,
                    pair0: int = 0, stream=None) -> None:
        n_pairs = y_cond.shape[0]
        _check(self.lib.mar_cfg_combine(self.handle, y_cond.data_ptr(), _ptr(y_uncond), pair0, n_pairs,
                                        op, float(scale), guided.data_ptr(), _ptr(uncond_out),
                                        _stream(stream)))

    def profile_start(self, kind: str) -> None:
        _check(self.lib.mar_profile_start(self.handle, PROF_KINDS.index(kind)))

    def profile_stop(self):
        """(ms_total, launches, flops, bytes) of the launches timed since start."""
        ms, n = ctypes.c_double(), ctypes.c_int64()
        fl, by = ctypes.c_double(), ctypes.c_double()
        _check(self.lib.mar_profile_stop(self.handle, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl),
                                         ctypes.byref(by)))
        return ms.value, n.value, fl.value, by.value

    def output(self):
        """The output cache [max_slots, S, D] fp32 as a view of the workspace."""
        torch = _torch()
        p = self.lib.mar_output(self.handle)
        off = p - self._ws.data_ptr()
        d = self.dims
        n = d.max_slots * d.seq_len * d.d_model
        return self._ws[off:off + 4 * n].view(torch.float32).view(d.max_slots, d.seq_len, d.d_model)


# --------------------------------------------------------------------------
# per-kernel entry points
# --------------------------------------------------------------------------

def k_layernorm(dtype: str, src, w, b, eps: float, out, idx=None, per_slot=None, seq=None,
                copy_f32=None, m=None, stream=None) -> None:
    torch = _torch()
    d = src.shape[-1]
    src_f32 = 1 if src.dtype == torch.float32 else 0
    if m is None:
        m = out.shape[0]
    if per_slot is None:
        per_slot = m if idx is None else idx.shape[-1]
    if seq is None:
        seq = per_slot
    _check(load().mar_k_layernorm(dtype_code(dtype), src.data_ptr(), src_f32, _ptr(idx), per_slot, seq, m, d,
                                  w.data_ptr(), b.data_ptr(), float(eps), _ptr(copy_f32), out.data_ptr(),
                                  _stream(stream)))


def k_linear(dtype: str, a, w, bias, out, gelu: bool = False, stream=None) -> None:
    m, k = a.shape
    n = w.shape[0]
    _check(load().mar_k_linear(dtype_code(dtype), 1 if gelu else 0, a.data_ptr(), w.data_ptr(),
                               bias.data_ptr(), m, n, k, out.data_ptr(), _stream(stream)))


def k_linear_residual(dtype: str, a, w, bias, resid, out, out_idx=None, per_slot=0, seq=0,
                      resid_copy=None, stream=None) -> None:
    m, k = a.shape
    n = w.shape[0]
    _check(load().mar_k_linear_residual(dtype_code(dtype), a.data_ptr(), w.data_ptr(), bias.data_ptr(), m,
                                        n, k, resid.data_ptr(), out.data_ptr(), _ptr(out_idx), per_slot,
                                        seq, _ptr(resid_copy), _stream(stream)))


def k_qkv(dtype: str, a, w, bias, d_model: int, n_heads: int, seq: int, per_slot: int,
          q_out=None, k_cache=None, v_cache=None, v_copy=None, idx=None, n_offset: int = 0,
          n_cols: Optional[int] = None, stream=None) -> None:
    m = a.shape[0]
    if n_cols is None:
        n_cols = w.shape[0]
    _check(load().mar_k_qkv(dtype_code(dtype), a.data_ptr(), w.data_ptr(), bias.data_ptr(), m, n_cols,
                            n_offset, d_model, n_heads, seq, per_slot, _ptr(idx), _ptr(q_out),
                            _ptr(k_cache), _ptr(v_cache), _ptr(v_copy), _stream(stream)))


def k_attention(dtype: str, q, k, v, out, n_slots: int, n_heads: int, seq: int, d_head: int,
                per_slot: int, stream=None) -> None:
    _check(load().mar_k_attention(dtype_code(dtype), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                  out.data_ptr(), n_slots, n_heads, seq, d_head, per_slot, _stream(stream)))


def k_scores(dtype: str, v_cur, v_ref, scores, update_ref: bool = False, stream=None) -> None:
    n_slots, n_heads, seq, d_head = v_cur.shape
    _check(load().mar_k_scores(dtype_code(dtype), v_cur.data_ptr(), v_ref.data_ptr(), n_slots, n_heads,
                               seq, d_head, scores.data_ptr(), 1 if update_ref else 0, _stream(stream)))


def k_select(scores, n: int, idx, stream=None, most_similar: bool = False) -> None:
    n_slots, seq = scores.shape
    fn = load().mar_k_select_most_similar if most_similar else load().mar_k_select
    _check(fn(scores.data_ptr(), n_slots, seq, n, idx.data_ptr(), _stream(stream)))


def k_gemm_variant(variant: int) -> None:
    """Force a tile configuration of the matrix products (-1: by shape)."""
    _check(load().mar_k_gemm_variant(variant))


# --------------------------------------------------------------------------
# rotary positions, the paged cache and its attention
# --------------------------------------------------------------------------

def _refuse(message: str) -> None:
    raise MarError(MAR_E_ARG, message)


def _dense(name: str, t, dtype, shape, device) -> None:
    """t is a dense tensor of this type and shape (None: any size) on `device`."""
    if t.dtype is not dtype or t.device != device or not t.is_contiguous():
        _refuse(f"{name}: need a contiguous {dtype} tensor on {device}, got {t.dtype} on {t.device}")
    have = t.shape
    if len(have) != len(shape) or (have != shape and any(n is not None and n != m for n, m in zip(shape, have))):
        _refuse(f"{name}: shape {tuple(have)} is not {shape}")


def _rows(name: str, t, dtype, m: int, d_head: int, device):
    """t is a matrix of m rows of whole heads on `device`, its columns dense:
    (heads, row stride).  A single row has no stride of its own and counts as
    dense."""
    shape, stride = t.shape, t.stride()
    if (t.dtype is dtype and len(shape) == 2 and shape[0] == m and d_head > 0 and not shape[1] % d_head
            and (stride[1] == 1 or shape[1] == 1) and t.device == device):
        return shape[1] // d_head, stride[0] if m > 1 else shape[1]
    _refuse(f"{name}: need {m} rows of whole heads of {d_head} dense columns, {dtype} on {device}, got {tuple(shape)} "
            f"with strides {stride}, {t.dtype} on {t.device}")


def _stream_here(device, stream) -> int:
    """The stream's handle; refuses tensors that are not on the current GPU."""
    torch = _torch()
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        _refuse(f"the tensors are on {device}: need the current GPU")
    if stream is not None:
        return stream.cuda_stream
    try:
        return torch._C._cuda_getCurrentRawStream(device.index)
    except AttributeError:
        return _stream()


def _int32(names: str, *sizes: int) -> None:
    """Refuses what ctypes would cut to 32 bits without a word.  (The calls ask
    only where any bit past 31 is set, which takes a fifth of the time.)"""
    if max(sizes) >= 2 ** 31 or min(sizes) < -2 ** 31:
        _refuse(f"{names} = {sizes}: more than 32 bits")


def _storage_code(dtype) -> int:
    torch = _torch()
    if dtype is torch.bfloat16:
        return MAR_BF16
    if dtype is not torch.float32:
        _refuse(f"unsupported storage type {dtype}")
    return MAR_F32


LAYOUTS = {"halves": MAR_ROTARY_HALVES, "neighbours": MAR_ROTARY_NEIGHBOURS}


def rotary_sections(sections: Sequence[int], base: float = 10000.0, shared: bool = False, device="cuda"):
    """(freq, axis) of `Rotary` for sections[a] pairs of axis a, one after the
    other: pair j of a section of n turns base^(-j / n) per position, as where
    every axis has the whole range of frequencies; with `shared` pair i of all P
    pairs turns base^(-i / P), as where the axes divide one range."""
    torch = _torch()
    P = sum(sections)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    power = [i / P for i in range(P)] if shared else [j / n for n in sections for j in range(n)]
    return (torch.tensor([base ** -p for p in power], dtype=torch.float64, device=device),
            torch.tensor(axis, dtype=torch.int32, device=device))


class Rotary:
    """Rotary positions: freq [pairs] fp64 (radians per position; negated ones
    turn back), axis [pairs] int32, layout "halves" (pair i is elements i and
    i + pairs) or "neighbours" (2 i and 2 i + 1)."""

    def __init__(self, freq, axis, n_axes: int, layout: str = "halves"):
        torch = _torch()
        if layout not in LAYOUTS:
            _refuse(f"unknown layout {layout!r}")
        _dense("freq", freq, torch.float64, (None,), freq.device)
        _dense("axis", axis, torch.int32, (freq.shape[0],), freq.device)
        _int32("pairs, n_axes", freq.shape[0], n_axes)
        self.freq, self.axis, self.n_axes = freq, axis, n_axes
        self.device = freq.device
        self.c = MarRotaryC(freq.data_ptr(), axis.data_ptr(), freq.shape[0], n_axes, LAYOUTS[layout])
        self.ref = ctypes.byref(self.c)


class MarPages:
    """The pages of a cache: k and v [n_pages, heads, page, d_head]."""

    def __init__(self, k, v):
        _storage_code(k.dtype)
        _dense("k", k, k.dtype, (None, None, None, None), k.device)
        _dense("v", v, k.dtype, tuple(k.shape), k.device)
        self.k, self.v = k, v


class PagedBatch:
    """Sequences that live in `pages`: table [seqs, max_pages], q_start [seqs +
    1] and kv_len [seqs], all int32.  The tensors are held and read at every
    call, so their contents may change from step to step; max_kv bounds every
    kv_len (None: what the table's row holds); the attention divides its work for
    that many keys, so a close bound is the faster one."""

    def __init__(self, pages: MarPages, table, q_start, kv_len, max_kv: Optional[int] = None):
        torch = _torch()
        dev = pages.k.device
        _dense("table", table, torch.int32, (None, None), dev)
        _dense("q_start", q_start, torch.int32, (table.shape[0] + 1,), dev)
        _dense("kv_len", kv_len, torch.int32, (table.shape[0],), dev)
        n_pages, heads, page, d_head = pages.k.shape
        if max_kv is None:
            max_kv = table.shape[1] * page
        _int32("pages' shape, table's shape, max_kv", *pages.k.shape, *table.shape, max_kv)
        self.pages, self.table, self.q_start, self.kv_len = pages, table, q_start, kv_len
        self.dtype, self.device, self.d_head, self.heads = pages.k.dtype, dev, d_head, heads
        self.code = _storage_code(pages.k.dtype)
        self.c = MarPagedBatchC(pages.k.data_ptr(), pages.v.data_ptr(), table.data_ptr(), q_start.data_ptr(),
                                kv_len.data_ptr(), n_pages, heads, page, d_head, table.shape[0], table.shape[1],
                                max_kv)
        self.ref = ctypes.byref(self.c)


def k_rotary(rotary: Rotary, x, pos, out, d_head: int, stream=None) -> None:
    """out = rotary positions pos [m, n_axes] int32 on the rows of x
    [m, heads * d_head]; out may be x."""
    m, dev, dtype = x.shape[0], rotary.device, x.dtype
    heads, ldx = _rows("x", x, dtype, m, d_head, dev)
    heads_out, ldo = _rows("out", out, dtype, m, d_head, dev)
    if heads_out != heads:
        _refuse("out and x differ in width")
    _dense("pos", pos, _torch().int32, (m, rotary.n_axes), dev)
    if (m | heads | d_head) >> 31:
        _int32("rows, heads, d_head", m, heads, d_head)
    _check(load().mar_k_rotary(_storage_code(dtype), rotary.ref, x.data_ptr(), ldx, pos.data_ptr(), m, heads, d_head,
                               out.data_ptr(), ldo, _stream_here(dev, stream)))


def k_paged_store(batch: PagedBatch, k, v, q=None, q_out=None, rotary: Optional[Rotary] = None, pos=None,
                  stream=None) -> None:
    """Keys k (rotated) and values v [m, heads * d_head] of the batch's new
    tokens into its pages; q, if given, rotated into q_out (which may be q)."""
    m, dev, dh, dtype = k.shape[0], batch.device, batch.d_head, batch.dtype
    heads_k, ldk = _rows("k", k, dtype, m, dh, dev)
    heads_v, ldv = _rows("v", v, dtype, m, dh, dev)
    if heads_k != batch.heads or heads_v != batch.heads:
        _refuse(f"k, v: need {batch.heads} heads of {dh}")
    heads = ldq = ldo = 0
    q_ptr = out_ptr = rot = pos_ptr = None
    if q is not None:
        if q_out is None:
            _refuse("q needs a q_out")
        heads, ldq = _rows("q", q, dtype, m, dh, dev)
        heads_out, ldo = _rows("q_out", q_out, dtype, m, dh, dev)
        if heads_out != heads:
            _refuse("q_out and q differ in width")
        q_ptr, out_ptr = q.data_ptr(), q_out.data_ptr()
    if rotary is not None:
        if pos is None or rotary.device != dev:
            _refuse("rotary needs pos, and its tables on the batch's GPU")
        _dense("pos", pos, _torch().int32, (m, rotary.n_axes), dev)
        rot, pos_ptr = rotary.ref, pos.data_ptr()
    if (m | heads) >> 31:
        _int32("rows, heads", m, heads)
    _check(load().mar_k_paged_store(batch.code, batch.ref, rot, pos_ptr, m, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                    heads, q_ptr, ldq, out_ptr, ldo, _stream_here(dev, stream)))


def paged_attention_workspace_bytes(batch: PagedBatch, m: int, n_heads_q: int, window: int = 0,
                                    sinks: int = 0) -> int:
    """Bytes of workspace that k_paged_attention makes use of for m rows."""
    _int32("m, n_heads_q, window, sinks", m, n_heads_q, window, sinks)
    lib = load()
    n = lib.mar_k_paged_attention_workspace_bytes(batch.code, batch.ref, m, n_heads_q, window, sinks)
    if n == 0 and lib.mar_last_error():
        raise MarError(MAR_E_ARG, lib.mar_last_error().decode())
    return n


def k_paged_attention(batch: PagedBatch, q, out, causal: bool = True, window: int = 0, sinks: int = 0,
                      workspace=None, stream=None) -> None:
    """Attention of the rows q [m, heads * d_head] over their sequences' tokens
    in the pages; workspace: a tensor of any type (see
    paged_attention_workspace_bytes) or None."""
    m, dev, dh, dtype = q.shape[0], batch.device, batch.d_head, batch.dtype
    heads, ldq = _rows("q", q, dtype, m, dh, dev)
    heads_out, ldo = _rows("out", out, dtype, m, dh, dev)
    if heads_out != heads:
        _refuse("out and q differ in width")
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        if workspace.device != dev or not workspace.is_contiguous():
            _refuse("workspace: need a contiguous tensor on the batch's GPU")
        ws_bytes = workspace.numel() * workspace.element_size()
        ws_ptr = workspace.data_ptr() if ws_bytes else None
    if (m | heads | window | sinks) >> 31:
        _int32("rows, heads, window, sinks", m, heads, window, sinks)
    _check(load().mar_k_paged_attention(batch.code, batch.ref, m, heads, q.data_ptr(), ldq, 1 if causal else 0, window,
                                        sinks, ws_ptr, ws_bytes, out.data_ptr(), ldo, _stream_here(dev, stream)))


# --------------------------------------------------------------------------
# drafted tokens
# --------------------------------------------------------------------------

def _missing(**named) -> None:
    """Refuses the first of the tensors that is None, if one is."""
    for name, t in named.items():
        if t is None:
            _refuse(f"{name} is missing")


def _vectors(device, i32, *named) -> None:
    """Each (name, tensor, n) is a dense vector of n int32 on `device`.  (A third of the
    time of one _dense each.)"""
    for name, t, n in named:
        if t is None:
            _missing(**{name: t})
        if t.dtype is not i32 or t.shape != (n,) or t.device != device or not t.is_contiguous():
            _dense(name, t, i32, (n,), device)


def _workspace(workspace, device):
    """(pointer, bytes) of a workspace tensor of any type, or of None."""
    if workspace is None:
        return None, 0
    if workspace.device != device or not workspace.is_contiguous():
        _refuse(f"workspace: need a contiguous tensor on {device}")
    n = workspace.numel() * workspace.element_size()
    return workspace.data_ptr() if n else None, n


def _vocab_rows(name: str, t, dtype, shape, device) -> int:
    """Row stride of t [m, vocab] with dense columns on `device` (a single row's
    counts as dense)."""
    have, stride = t.shape, t.stride()
    if t.dtype is dtype and have == shape and (stride[1] == 1 or have[1] == 1) and t.device == device:
        return stride[0] if have[0] > 1 else have[1]
    _refuse(f"{name}: need {tuple(shape)} with dense columns, {dtype} on {device}, got {tuple(have)} with strides "
            f"{stride}, {t.dtype} on {t.device}")


def paged_tree_attention_workspace_bytes(batch: PagedBatch, m: int, n_heads_q: int, window: int = 0,
                                         sinks: int = 0) -> int:
    """Bytes of workspace that k_paged_tree_attention makes use of for m rows."""
    _int32("m, n_heads_q, window, sinks", m, n_heads_q, window, sinks)
    lib = load()
    n = lib.mar_k_paged_tree_attention_workspace_bytes(batch.code, batch.ref, m, n_heads_q, window, sinks)
    if n == 0 and lib.mar_last_error():
        raise MarError(MAR_E_ARG, lib.mar_last_error().decode())
    return n


def k_paged_tree_attention(batch: PagedBatch, q, parent, out, window: int = 0, sinks: int = 0, workspace=None,
                           stream=None) -> None:
    """Attention of the rows q [m, heads * d_head], the nodes of their sequences'
    trees (parent [m] int32: number of a row's parent in its sequence, or -1), over
    the past, themselves and their ancestors."""
    if q is None or out is None:
        _missing(q=q, out=out)
    m, dev, dh, dtype = q.shape[0], batch.device, batch.d_head, batch.dtype
    heads, ldq = _rows("q", q, dtype, m, dh, dev)
    heads_out, ldo = _rows("out", out, dtype, m, dh, dev)
    if heads_out != heads:
        _refuse("out and q differ in width")
    _vectors(dev, batch.kv_len.dtype, ("parent", parent, m))
    ws_ptr, ws_bytes = _workspace(workspace, dev)
    if (m | heads | window | sinks) >> 31:
        _int32("rows, heads, window, sinks", m, heads, window, sinks)
    _check(load().mar_k_paged_tree_attention(batch.code, batch.ref, m, heads, q.data_ptr(), ldq, parent.data_ptr(),
                                             window, sinks, ws_ptr, ws_bytes, out.data_ptr(), ldo,
                                             _stream_here(dev, stream)))


def k_probabilities(logits, out, temperature=None, stream=None) -> None:
    """out [m, vocab] fp32 = probabilities of the logits' rows at temperature [m]
    fp32 (None: 1; 0: one at the first largest logit)."""
    torch = _torch()
    if logits is None or out is None:
        _missing(logits=logits, out=out)
    dev, dtype, shape = logits.device, logits.dtype, logits.shape
    if len(shape) != 2:
        _refuse(f"logits: need [m, vocab], got {tuple(shape)}")
    ld = _vocab_rows("logits", logits, dtype, shape, dev)
    ldo = _vocab_rows("out", out, torch.float32, shape, dev)
    m, vocab = shape
    if temperature is not None:
        _dense("temperature", temperature, torch.float32, (m,), dev)
    if (m | vocab) >> 31:
        _int32("logits' shape", m, vocab)
    _check(load().mar_k_probabilities(_storage_code(dtype), logits.data_ptr(), ld, _ptr(temperature), m, vocab,
                                      out.data_ptr(), ldo, _stream_here(dev, stream)))


def draft_verify_workspace_bytes(m: int, n_seqs: int, vocab: int) -> int:
    """Bytes of workspace that k_draft_verify needs."""
    _int32("m, n_seqs, vocab", m, n_seqs, vocab)
    lib = load()
    n = lib.mar_k_draft_verify_workspace_bytes(m, n_seqs, vocab)
    if n == 0 and lib.mar_last_error():
        raise MarError(MAR_E_ARG, lib.mar_last_error().decode())
    return n


def k_draft_verify(q_start, p, parent, tokens, path, kept, next_token, random=None, draft=None, workspace=None,
                   stream=None) -> None:
    """Which nodes of the trees [q_start[s], q_start[s + 1]) the probabilities p [m,
    vocab] keep: path [m], kept [n_seqs], and next_token [n_seqs] after them.
    random [m] fp32: a number in [0, 1) per node, node 0's for the next token
    (None: greedy); draft [m, vocab]: probabilities that a node's children were
    drawn from (None: they are proposed as they are)."""
    torch = _torch()
    if p is None or q_start is None:
        _missing(p=p, q_start=q_start)
    dev, dtype, shape = p.device, p.dtype, p.shape
    if len(shape) != 2 or len(q_start.shape) != 1 or q_start.shape[0] < 1:
        _refuse("need p [m, vocab] and q_start [n_seqs + 1]")
    ldp = _vocab_rows("p", p, dtype, shape, dev)
    ldd = _vocab_rows("draft", draft, dtype, shape, dev) if draft is not None else 0
    m, vocab = shape
    n_seqs, i32 = q_start.shape[0] - 1, torch.int32
    _vectors(dev, i32, ("q_start", q_start, n_seqs + 1), ("parent", parent, m), ("tokens", tokens, m),
             ("path", path, m), ("kept", kept, n_seqs), ("next_token", next_token, n_seqs))
    if random is not None:
        _dense("random", random, torch.float32, (m,), dev)
    ws_ptr, ws_bytes = _workspace(workspace, dev)
    if (m | vocab | n_seqs) >> 31:
        _int32("m, vocab, n_seqs", m, vocab, n_seqs)
    _check(load().mar_k_draft_verify(_storage_code(dtype), n_seqs, q_start.data_ptr(), m, vocab, p.data_ptr(), ldp,
                                     _ptr(draft), ldd, parent.data_ptr(), tokens.data_ptr(), _ptr(random),
                                     path.data_ptr(), kept.data_ptr(), next_token.data_ptr(), ws_ptr, ws_bytes,
                                     _stream_here(dev, stream)))


def k_paged_keep(batch: PagedBatch, path, kept, kv_len_out, stream=None) -> None:
    """The kept nodes' keys and values (path [m], kept [seqs] as k_draft_verify
    leaves them) moved together in the batch's pages; kv_len_out [seqs]: the
    lengths that remain."""
    dev, i32, n = batch.device, batch.kv_len.dtype, batch.c.n_seqs
    if path is None:
        _missing(path=path)
    m = path.shape[0] if len(path.shape) == 1 else -1
    _vectors(dev, i32, ("path", path, m), ("kept", kept, n), ("kv_len_out", kv_len_out, n))
    if m >> 31:
        _int32("rows", m)
    _check(load().mar_k_paged_keep(batch.code, batch.ref, m, path.data_ptr(), kept.data_ptr(), kv_len_out.data_ptr(),
                                   _stream_here(dev, stream)))


def paged_fork_workspace_bytes(batch: PagedBatch, n_new: int) -> int:
    """Bytes of workspace that k_paged_fork needs for n_new rows."""
    _int32("n_new", n_new)
    lib = load()
    n = lib.mar_k_paged_fork_workspace_bytes(batch.ref, n_new)
    if n == 0:
        raise MarError(MAR_E_ARG, lib.mar_last_error().decode())
    return n


def k_paged_fork(batch: PagedBatch, source, table_out, kv_len_out, missing, keep=None, add=None, workspace=None,
                 stream=None) -> None:
    """A new table: row i continues sequence source[i] with its first keep[i]
    tokens (None: all) and room for add[i] more (None: none).  table_out [n,
    max_pages], kv_len_out [n], missing [1]; source, keep, add [n]; all int32."""
    dev, i32 = batch.device, batch.kv_len.dtype
    if source is None or table_out is None:
        _missing(source=source, table_out=table_out)
    n = source.shape[0] if len(source.shape) == 1 else -1
    _vectors(dev, i32, ("source", source, n), ("kv_len_out", kv_len_out, n), ("missing", missing, 1))
    if keep is not None:
        _vectors(dev, i32, ("keep", keep, n))
    if add is not None:
        _vectors(dev, i32, ("add", add, n))
    _dense("table_out", table_out, i32, (n, batch.c.max_pages), dev)
    ws_ptr, ws_bytes = _workspace(workspace, dev)
    if n >> 31:
        _int32("rows", n)
    _check(load().mar_k_paged_fork(batch.code, batch.ref, n, source.data_ptr(), _ptr(keep), _ptr(add),
                                   table_out.data_ptr(), kv_len_out.data_ptr(), missing.data_ptr(), ws_ptr, ws_bytes,
                                   _stream_here(dev, stream)))


# --------------------------------------------------------------------------
# the diffusion head (include/mar_head.h)
# --------------------------------------------------------------------------

def head_dims_c(hd) -> MarHeadDimsC:
    return MarHeadDimsC(hd.width, hd.depth, hd.cond_dim, hd.token_dim, hd.steps, hd.train_steps, hd.freq_dim,
                        hd.max_rows, dtype_code(hd.dtype), hd.beta_start, hd.beta_end, hd.ln_eps)


def head_workspace_bytes(hd) -> int:
    d = head_dims_c(hd)
    n = load().mar_head_workspace_bytes(ctypes.byref(d))
    if n == 0:
        raise MarError(MAR_E_SHAPE, load().mar_last_error().decode())
    return n


class MarHead:
    """Handle over a workspace tensor; the library copies the head's weights
    in and computes its time embeddings."""

    def __init__(self, hd, weights: Dict[str, "object"], device="cuda", stream=None):
        torch = _torch()
        self.dims = hd
        self.lib = load()
        nbytes = head_workspace_bytes(hd)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.workspace.data_ptr()) % 256
        self._ws = self.workspace[off:off + nbytes]
        w = MarHeadWeightsC(*[weights[f].data_ptr() for f in HEAD_WEIGHT_FIELDS])
        self._weights = weights
        handle = ctypes.c_void_p()
        d = head_dims_c(hd)
        _check(self.lib.mar_head_init(ctypes.byref(d), ctypes.byref(w), self._ws.data_ptr(), nbytes,
                                      _stream(stream), ctypes.byref(handle)))
        self.handle = handle

    def close(self) -> None:
        if getattr(self, "handle", None):
            self.lib.mar_head_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sample(self, y_cond, y_uncond, row_cond, row_uncond, x_init, xi, scale: float, x_out,
               trajectory=None, eps_out=None, stream=None, noalloc: bool = False) -> None:
        """y_cond, y_uncond: [y_rows, cond_dim] fp32 (any leading shape
        flattened); row_*: int32 [rows]; x_init [rows, T]; xi [steps, rows, T].
        noalloc: the entry point whose scratch is the library's static array."""
        y_rows = y_cond.numel() // self.dims.cond_dim
        fn = self.lib.mar_head_sample_noalloc if noalloc else self.lib.mar_head_sample
        _check(fn(self.handle, y_cond.data_ptr(), y_uncond.data_ptr(), y_rows,
                                        row_cond.data_ptr(), row_uncond.data_ptr(), row_cond.shape[0],
                                        x_init.data_ptr(), xi.data_ptr(), float(scale), x_out.data_ptr(),
                                        _ptr(trajectory), _ptr(eps_out), _stream(stream)))
