"""Python binding of the gfx950 sparse INT8 linear library (libsparse_linear.so).

Argument marshalling only: every step of the layer runs in the library's HIP
kernels. PyTorch is used for device memory and streams. There is no CPU or
PyTorch fallback: if the shared library is missing, ``load()`` raises.

    import paper_2211_07715_amd as sl
    pw = sl.PackedWeight.pack(w_int8, w_scale, bias)        # host -> device, once
    q = sl.quantize_act(x_f32_cuda, x_scale)                 # first op of a chain
    y = pw.run(q, x_scale, sl.EPI_I8_GELU, out_scale=so)     # int8 [M, N]

Activations between layers can stay in the 16-token x 32-feature block layout
(LAYOUT_T16X32, 4-D tensors [ceil(M/16), ceil(C/32), 16, 32]), the order the
matrix cores read them in:

    q = sl.quantize_act(x_f32_cuda, x_scale, layout=sl.LAYOUT_T16X32)
    h = pw1.run(q, x_scale, sl.EPI_I8_GELU, out_scale=so, m_tokens=M,
                x_layout=sl.LAYOUT_T16X32, y_layout=sl.LAYOUT_T16X32)
    y = pw2.run(h, so, sl.EPI_F32, m_tokens=M, x_layout=sl.LAYOUT_T16X32)   # fp32 [M, N2]

Between the linears of an encoder layer (a batch's sequences one after the other
in the token dimension, seq_start their first tokens and the end):

    a = sl.attention(qkv, s_qkv, seq_start, max_len, n_heads, head_dim, out_scale=s_a)      # int8 -> int8
    blocks = sl.select_blocks(qkv, seq_start, max_len, n_heads, head_dim, top_k)            # long sequences:
    a = sl.attention(qkv, s_qkv, seq_start, max_len, n_heads, head_dim, out_scale=s_a, blocks=blocks)
    _, u, q = sl.residual_norm(y, gamma, beta, residual=x, keep_norm=True, out_scale=s_q)   # LayerNorm(x + y)

In a decoder, with an int8 cache of keys and values in pages (kv_len: a sequence's
cached tokens with the call's own; page_table: the numbers of its pages):

    cache = torch.zeros(sl.cache_shape(n_pages, page_size, n_kv_heads, head_dim), dtype=torch.int8, device="cuda")
    q = sl.cache_append(qkv, cache, page_table, seq_start, kv_len, max_new, n_heads, x_scale=s_qkv, q_scale=s_q,
                        k_scale=s_k, v_scale=s_v, rope=sl.ROPE_HALF, inv_freq=inv_freq)
    a = sl.cache_attention(q, cache, page_table, seq_start, kv_len, max_new, max_len, n_heads, q_scale=s_q,
                           k_scale=s_k, v_scale=s_v, out_scale=s_a)      # causal=False: over an encoder's states

Calls run on the current stream, or on `stream`: the caller then orders it behind
what makes the inputs and before what reads the results. Memory that a call
allocates for results is that stream's.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsparse_linear.so")

EPI_ACC_I32, EPI_F32, EPI_F32_GELU, EPI_I8, EPI_I8_GELU = 0, 1, 2, 3, 4
EPI_BY_NAME = {"acc_i32": 0, "f32": 1, "f32_gelu": 2, "i8": 3, "i8_gelu": 4}
LAYOUT_ROWS, LAYOUT_T16X32 = 0, 1
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_ELEMENT = 0, 1, 2, 3
ACT_NONE, ACT_F32, ACT_I8 = 0, 1, 2
ROPE_NONE, ROPE_HALF, ROPE_INTERLEAVED = 0, 1, 2
KEY_BLOCK = 64  # keys of a selectable block

SL_OK = 0
STATUS = {0: "SL_OK", -1: "SL_ERR_INVALID_ARG", -2: "SL_ERR_SHAPE", -3: "SL_ERR_HIP", -4: "SL_ERR_OOM",
          -5: "SL_ERR_UNSUPPORTED", -6: "SL_ERR_NOT_ON_DEVICE"}

# every symbol include/sparse_linear.h declares
EXPORTS = ("sparse_linear_pack", "sparse_linear_pack_host", "sparse_linear_run", "sparse_linear_run_layout",
           "quantize_act", "quantize_act_layout", "residual_norm", "attention_run", "attention_select",
           "attention_select_workspace", "cache_append", "cache_attention", "cache_attention_workspace",
           "sparse_linear_unpack", "sparse_linear_info", "sparse_linear_export_bsr",
           "sparse_linear_tile_stats", "sparse_linear_free", "sl_status_string", "sl_last_error",
           "sl_abi_version", "sl_last_path", "sl_reload_env", "sl_gelu_table_codes")

# kernel-selection overrides the library reads from the environment
ENV_KEYS = ("SL_PATH", "SL_TILE", "SL_DTILE", "SL_PTILE", "SL_PSLICES")
_env_seen: Optional[tuple] = None
_env_getters: Optional[tuple] = None

_lib: Optional[ctypes.CDLL] = None


class SparseLinearError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: {STATUS.get(status, status)}: {detail}")
        self.status = status


def load() -> ctypes.CDLL:
    """Load the in-tree shared library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2211_07715_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    pp = ctypes.POINTER(ctypes.c_void_p)
    lib.sparse_linear_pack.argtypes = [vp, i32, i32, i32, i32, vp, vp, pp]
    lib.sparse_linear_pack_host.argtypes = [vp, i32, i32, i32, i32, vp, vp, pp]
    lib.sparse_linear_run.argtypes = [vp, vp, i64, f32, i32, f32, vp, vp]
    lib.sparse_linear_run_layout.argtypes = [vp, vp, i32, i64, f32, i32, f32, vp, i32, vp]
    lib.quantize_act.argtypes = [vp, i64, f32, vp, vp]
    lib.quantize_act_layout.argtypes = [vp, i64, i32, f32, vp, i32, vp]
    lib.residual_norm.argtypes = [vp, vp]
    lib.attention_run.argtypes = [vp, vp]
    lib.attention_select.argtypes = [vp, vp, vp, i64, vp]
    lib.attention_select_workspace.argtypes = [vp]
    lib.attention_select_workspace.restype = i64
    lib.cache_append.argtypes = [vp, vp]
    lib.cache_attention.argtypes = [vp, vp]
    lib.cache_attention_workspace.argtypes = [vp]
    lib.cache_attention_workspace.restype = i64
    lib.sparse_linear_unpack.argtypes = [vp, vp]
    lib.sparse_linear_info.argtypes = [vp, vp, vp, vp]
    lib.sparse_linear_export_bsr.argtypes = [vp, vp, vp, vp]
    lib.sparse_linear_tile_stats.argtypes = [vp, vp, vp, vp, vp]
    for name in ("sparse_linear_pack", "sparse_linear_pack_host", "sparse_linear_run", "sparse_linear_run_layout",
                 "quantize_act", "quantize_act_layout", "residual_norm", "attention_run", "attention_select",
                 "cache_append", "cache_attention", "sparse_linear_unpack", "sparse_linear_info", "sparse_linear_export_bsr",
                 "sparse_linear_tile_stats"):
        getattr(lib, name).restype = i32
    lib.sparse_linear_free.argtypes = [vp]
    lib.sparse_linear_free.restype = None
    lib.sl_status_string.argtypes = [i32]
    lib.sl_status_string.restype = ctypes.c_char_p
    lib.sl_last_error.argtypes = []
    lib.sl_last_error.restype = ctypes.c_char_p
    lib.sl_abi_version.argtypes = []
    lib.sl_abi_version.restype = i32
    lib.sl_last_path.argtypes = []
    lib.sl_last_path.restype = ctypes.c_char_p
    lib.sl_reload_env.argtypes = []
    lib.sl_reload_env.restype = None
    lib.sl_gelu_table_codes.argtypes = [f32, vp, vp, i64]
    lib.sl_gelu_table_codes.restype = i32
    _lib = lib
    return lib


def _sync_env(lib: ctypes.CDLL):
    """The library reads SL_PATH / SL_*TILE once; have it read them again when
    this process has changed them since the last run."""
    global _env_seen, _env_getters
    # (os.environ encodes and decodes on every read, 0.4 us a key: the mapping
    # of encoded names that it keeps is read where there is one)
    if _env_getters is None or _env_getters[0] is not os.environ:
        data = getattr(os.environ, "_data", None)
        keys = tuple(os.fsencode(k) for k in ENV_KEYS)
        if type(data) is dict and all(isinstance(k, bytes) for k in data):
            _env_getters = (os.environ, data.get, *keys)
        else:
            _env_getters = (os.environ, os.environ.get, *ENV_KEYS)
    _, get, k0, k1, k2, k3, k4 = _env_getters
    now = (get(k0), get(k1), get(k2), get(k3), get(k4))
    if now != _env_seen:
        lib.sl_reload_env()
        _env_seen = now


def _check(status: int, where: str):
    if status != SL_OK:
        detail = load().sl_last_error().decode(errors="replace")
        raise SparseLinearError(status, where, detail)


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def t16x32_shape(rows: int, cols: int):
    """Shape of a [rows x cols] activation in LAYOUT_T16X32."""
    return ((rows + 15) // 16, (cols + 31) // 32, 16, 32)


def to_t16x32(a: np.ndarray, fill: int = 0) -> np.ndarray:
    """Host copy of an int8 [rows x cols] array in LAYOUT_T16X32 (padding = fill)."""
    rows, cols = a.shape
    rb, cb, _, _ = t16x32_shape(rows, cols)
    p = np.full((rb * 16, cb * 32), fill, dtype=a.dtype)
    p[:rows, :cols] = a
    return np.ascontiguousarray(p.reshape(rb, 16, cb, 32).transpose(0, 2, 1, 3))


def from_t16x32(b: np.ndarray, rows: int, cols: int) -> np.ndarray:
    """The [rows x cols] array held by a LAYOUT_T16X32 array (padding dropped)."""
    rb, cb, _, _ = b.shape
    return np.ascontiguousarray(b.transpose(0, 2, 1, 3).reshape(rb * 16, cb * 32)[:rows, :cols])


_torch = None      # set by _torch_once()
_raw_stream = None  # () -> the current device's current stream, as an integer
_KIND_DTYPE: dict = {}


def _torch_once():
    """Import torch at the first call that needs it, and look up once what every call asks it for."""
    global _torch, _raw_stream
    import torch
    _KIND_DTYPE.update({EPI_ACC_I32: torch.int32, EPI_F32: torch.float32, EPI_F32_GELU: torch.float32,
                        EPI_I8: torch.int8, EPI_I8_GELU: torch.int8})
    # torch.cuda.current_stream() makes a Stream object to hold the number that
    # torch's own launches read directly (3.2 against 0.2 us a call)
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and device is not None:
        _raw_stream = lambda: raw(device())
    else:
        _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    _torch = torch
    return torch


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        _torch_once()
    return _raw_stream()


def _empty(shape, dtype, device, stream):
    """Memory of a result that `stream` (None: the current one) writes. For another stream than the current one it is of
    that stream's, where no earlier work of the current one is on it, and is not handed on before the current one's later
    work on it."""
    if stream is None or stream.cuda_stream == _raw_stream():
        return _torch.empty(shape, dtype=dtype, device=device)
    current = _torch.cuda.current_stream(device)
    with _torch.cuda.stream(stream):
        out = _torch.empty(shape, dtype=dtype, device=device)
    out.record_stream(current)
    return out


class PackedWeight:
    """An immutable packed 4x1 block-sparse int8 weight (one C handle)."""

    def __init__(self, handle: int, n_out: int, k_in: int, on_device: bool):
        self._h = ctypes.c_void_p(handle)
        self.n_out = n_out
        self.k_in = k_in
        self.on_device = on_device

    @classmethod
    def pack(cls, w: np.ndarray, w_scale: np.ndarray, bias: Optional[np.ndarray] = None,
             host_only: bool = False) -> "PackedWeight":
        lib = load()
        w = np.ascontiguousarray(w, dtype=np.int8)
        if w.ndim != 2:
            raise ValueError("w must be [n_out, k_in]")
        sw = np.ascontiguousarray(w_scale, dtype=np.float32)
        b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
        n, k = w.shape
        if sw.shape != (n,) or (b is not None and b.shape != (n,)):
            raise ValueError("w_scale and bias must have shape [n_out]")
        h = ctypes.c_void_p()
        fn = lib.sparse_linear_pack_host if host_only else lib.sparse_linear_pack
        _check(fn(_np_ptr(w), n, k, 4, 1, _np_ptr(sw), _np_ptr(b), ctypes.byref(h)), fn.__name__)
        return cls(h.value, n, k, not host_only)

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise ValueError("packed weight was freed")
        return self._h

    def free(self):
        if self._h:
            load().sparse_linear_free(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def info(self):
        n, k, nnzb = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int64()
        _check(load().sparse_linear_info(self.handle, ctypes.byref(n), ctypes.byref(k), ctypes.byref(nnzb)),
               "sparse_linear_info")
        return n.value, k.value, nnzb.value

    def nnz_blocks(self) -> int:
        return self.info()[2]

    def unpack(self) -> np.ndarray:
        out = np.empty((self.n_out, self.k_in), dtype=np.int8)
        _check(load().sparse_linear_unpack(self.handle, _np_ptr(out)), "sparse_linear_unpack")
        return out

    def export_bsr(self):
        nnzb = self.nnz_blocks()
        row_ptr = np.empty(self.n_out // 4 + 1, dtype=np.uint32)
        col = np.empty(nnzb, dtype=np.uint16)
        vals = np.empty((nnzb, 4), dtype=np.int8)
        _check(load().sparse_linear_export_bsr(self.handle, _np_ptr(row_ptr), _np_ptr(col), _np_ptr(vals)),
               "sparse_linear_export_bsr")
        return row_ptr, col, vals

    def tile_stats(self):
        nt, ne, no, ib = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        _check(load().sparse_linear_tile_stats(self.handle, ctypes.byref(nt), ctypes.byref(ne), ctypes.byref(no),
                                               ctypes.byref(ib)), "sparse_linear_tile_stats")
        return {"n_tiles": nt.value, "n_entries": ne.value, "n_overflow": no.value, "image_bytes": ib.value}

    def run(self, x, x_scale: float, kind: int, out_scale: float = 1.0, out=None, stream=None,
            x_layout: int = LAYOUT_ROWS, y_layout: int = LAYOUT_ROWS, m_tokens: Optional[int] = None):
        """Y = epilogue(X W^T) for a CUDA int8 tensor x; returns Y.

        x: [M, k_in] (LAYOUT_ROWS) or t16x32_shape(M, k_in) with m_tokens=M
        (LAYOUT_T16X32). Y: [M, n_out] of the kind's dtype, or, for the int8
        kinds with y_layout=LAYOUT_T16X32, t16x32_shape(M, n_out) int8."""
        torch = _torch or _torch_once()
        if x.dtype != torch.int8 or not x.is_cuda or not x.is_contiguous():
            raise ValueError("x must be a contiguous CUDA int8 tensor")
        if x_layout == LAYOUT_ROWS:
            if x.dim() != 2 or x.shape[1] != self.k_in:
                raise ValueError(f"x must be [M, {self.k_in}]")
            m = x.shape[0] if m_tokens is None else int(m_tokens)
            if m != x.shape[0]:
                raise ValueError("m_tokens differs from x's rows")
        elif x_layout == LAYOUT_T16X32:
            if m_tokens is None:
                raise ValueError("m_tokens is required with LAYOUT_T16X32 input")
            m = int(m_tokens)
            if tuple(x.shape) != t16x32_shape(m, self.k_in):
                raise ValueError(f"x must have shape {t16x32_shape(m, self.k_in)}")
        else:
            raise ValueError(f"unknown x_layout {x_layout}")
        dt = _KIND_DTYPE[kind]
        shape = t16x32_shape(m, self.n_out) if y_layout == LAYOUT_T16X32 else (m, self.n_out)
        if out is None:
            out = _empty(shape, dt, x.device, stream)
        elif out.dtype != dt or tuple(out.shape) != tuple(shape) or not out.is_contiguous():
            raise ValueError("out has the wrong dtype/shape or is not contiguous")
        lib = load()
        _sync_env(lib)
        st = lib.sparse_linear_run_layout(self.handle, x.data_ptr(), int(x_layout), m, float(x_scale), int(kind),
                                          float(out_scale), out.data_ptr(), int(y_layout), _stream_ptr(stream))
        if st != SL_OK:
            _check(st, "sparse_linear_run_layout")
        return out


def last_path() -> str:
    """Kernel and workgroup shape of the last successful run (of a linear or of either attention) on this thread."""
    return load().sl_last_path().decode()


def gelu_table_codes(out_scale: float, y: np.ndarray) -> Optional[np.ndarray]:
    """int8 codes of the GELU + requantisation step table for fp32 values y,
    looked up as the kernels do; None when out_scale admits no table."""
    lib = load()
    y = np.ascontiguousarray(y, dtype=np.float32)
    q = np.empty(y.shape, dtype=np.int8)
    st = lib.sl_gelu_table_codes(float(out_scale), _np_ptr(y), _np_ptr(q), y.size)
    if st == -5:
        return None
    _check(st, "sl_gelu_table_codes")
    return q


def quantize_act(x, scale: float, out=None, stream=None, layout: int = LAYOUT_ROWS):
    """q = clamp(rint(x / scale), -127, 127) for a contiguous CUDA fp32 tensor:
    same shape (LAYOUT_ROWS), or, for a 2-D x [rows, cols] and
    layout=LAYOUT_T16X32, int8 of shape t16x32_shape(rows, cols)."""
    torch = _torch or _torch_once()
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA float32 tensor")
    if layout == LAYOUT_ROWS:
        if out is None:
            out = _empty(x.shape, torch.int8, x.device, stream)
        elif out.dtype != torch.int8 or out.numel() != x.numel() or not out.is_contiguous():
            raise ValueError("out must be a contiguous int8 tensor with x's size")
        _check(load().quantize_act(x.data_ptr(), x.numel(), float(scale), out.data_ptr(), _stream_ptr(stream)),
               "quantize_act")
        return out
    if layout != LAYOUT_T16X32 or x.dim() != 2:
        raise ValueError("LAYOUT_T16X32 quantisation takes a 2-D x [rows, cols]")
    rows, cols = x.shape
    shape = t16x32_shape(rows, cols)
    if out is None:
        out = _empty(shape, torch.int8, x.device, stream)
    elif out.dtype != torch.int8 or tuple(out.shape) != shape or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous int8 tensor of shape {shape}")
    _check(load().quantize_act_layout(x.data_ptr(), rows, cols, float(scale), out.data_ptr(), int(layout),
                                      _stream_ptr(stream)),
           "quantize_act_layout")
    return out


# --- between the linears ------------------------------------------------------

# sl_residual_norm_args, sl_attention_args, sl_cache_append_args and sl_cache_attention_args, field by field
_NORM_ARGS = struct.Struct("q10P9i5f0q")
_ATTN_ARGS = struct.Struct("Pq4P10i3f0q")
_APPEND_ARGS = struct.Struct("Pq7P13i5f0q")
_CACHE_ARGS = struct.Struct("Pq6Pq14i5f0q")


def _act_type(x, name: str, layout: int, shape) -> int:
    """ACT_F32 or ACT_I8 of a CUDA activation tensor that holds [rows, cols] = shape."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    dt = x.dtype
    if dt is _torch.float32:
        if x.shape != shape:  # (a torch.Size is a tuple)
            raise ValueError(f"{name} must be {shape}")
        return ACT_F32
    if dt is not _torch.int8:
        raise ValueError(f"{name} must be float32 or int8")
    want = t16x32_shape(*shape) if layout == LAYOUT_T16X32 else shape
    if x.shape != want:
        raise ValueError(f"{name} must have shape {want}")
    return ACT_I8


def _f32_ptr(x, name: str, shape) -> int:
    """Address of a contiguous fp32 CUDA tensor of that shape."""
    if x.dtype is not _torch.float32 or x.shape != shape or not x.is_cuda or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor of shape {shape}")
    return x.data_ptr()


def residual_norm(y, gamma=None, beta=None, *, norm: int = NORM_LAYER, eps: float = 1e-12, y_scale: float = 1.0,
                  residual=None, residual_scale: float = 1.0, r_scale: float = 1.0, gate=None,
                  post_norm: int = NORM_NONE, post_gamma=None, post_beta=None, keep_sum=False, keep_norm=False,
                  out_scale: Optional[float] = None, y_layout: int = LAYOUT_ROWS, r_layout: int = LAYOUT_ROWS,
                  q_layout: int = LAYOUT_ROWS, shape=None, q_out=None, stream=None):
    """The boundary between two blocks of a layer, in one pass:

        t = post_norm(y);  h = residual_scale * residual + gate * t;  u = norm(h);  q = codes of u / out_scale

    y, residual: fp32 [rows, cols], or int8 codes (of y_scale, r_scale) in
    y_layout / r_layout; block-layout tensors need shape=(rows, cols). gate: fp32
    [cols], [rows, 1] or [rows, cols]. Returns (h, u, q): h where keep_sum, u
    where keep_norm (True, or a fp32 tensor to write to, which may be y or
    residual itself), q (int8, q_layout) where out_scale is given; None for the
    others."""
    torch = _torch or _torch_once()
    if shape is None:
        if y.dim() != 2:
            raise ValueError("shape=(rows, cols) is needed for a y in the block layout")
        shape = y.shape
    shape = rows, cols = int(shape[0]), int(shape[1])
    y_type = _act_type(y, "y", y_layout, shape)
    r_type = ACT_NONE if residual is None else _act_type(residual, "residual", r_layout, shape)
    gate_kind, gate_ptr = GATE_NONE, 0
    if gate is not None:
        gs = gate.shape
        gate_kind = (GATE_CHANNEL if gs == (cols,) else GATE_ELEMENT if gs == shape and cols > 1 else
                     GATE_TOKEN if gs == (rows, 1) else -1)
        if gate_kind < 0:
            raise ValueError(f"gate must be [{cols}], [{rows}, 1] or [{rows}, {cols}]")
        gate_ptr = _f32_ptr(gate, "gate", gs)
    channels = (cols,)
    h = u = q = None
    if keep_sum is not False and keep_sum is not None:
        h = _empty(shape, torch.float32, y.device, stream) if keep_sum is True else keep_sum
    if keep_norm is not False and keep_norm is not None:
        u = _empty(shape, torch.float32, y.device, stream) if keep_norm is True else keep_norm
    if out_scale is not None:
        q_shape = t16x32_shape(rows, cols) if q_layout == LAYOUT_T16X32 else shape
        if q_out is None:
            q = _empty(q_shape, torch.int8, y.device, stream)
        else:
            q = q_out
            if q.dtype is not torch.int8 or q.shape != q_shape or not q.is_contiguous() or not q.is_cuda:
                raise ValueError(f"q_out must be a contiguous CUDA int8 tensor of shape {q_shape}")
    args = _NORM_ARGS.pack(
        rows, y.data_ptr(), 0 if residual is None else residual.data_ptr(), gate_ptr,
        0 if post_gamma is None else _f32_ptr(post_gamma, "post_gamma", channels),
        0 if post_beta is None else _f32_ptr(post_beta, "post_beta", channels),
        0 if gamma is None else _f32_ptr(gamma, "gamma", channels),
        0 if beta is None else _f32_ptr(beta, "beta", channels),
        0 if h is None else _f32_ptr(h, "keep_sum", shape), 0 if u is None else _f32_ptr(u, "keep_norm", shape),
        0 if q is None else q.data_ptr(), cols, y_type, y_layout, r_type, r_layout, gate_kind, post_norm, norm, q_layout,
        y_scale, r_scale, residual_scale, eps, 1.0 if out_scale is None else out_scale)
    st = load().residual_norm(args, _stream_ptr(stream))
    if st != SL_OK:
        _check(st, "residual_norm")
    return h, u, q


def _attention_args(x, seq_start, max_len, n_heads, head_dim, n_kv_heads, key_len, x_layout, m_tokens):
    """Checks of what attention and select_blocks share; returns (m_tokens, n_kv_heads, n_seq)."""
    torch = _torch or _torch_once()
    n_kv = n_heads if n_kv_heads is None else n_kv_heads
    if head_dim < 1:
        raise ValueError("head_dim must be >= 1")
    cols = (n_heads + 2 * n_kv) * head_dim
    if x.dtype != torch.int8 or not x.is_cuda or not x.is_contiguous():
        raise ValueError("qkv must be a contiguous CUDA int8 tensor")
    if x_layout == LAYOUT_T16X32:
        if m_tokens is None:
            raise ValueError("m_tokens is required with LAYOUT_T16X32 input")
        if tuple(x.shape) != t16x32_shape(m_tokens, cols):
            raise ValueError(f"qkv must have shape {t16x32_shape(m_tokens, cols)}")
    elif x.dim() != 2 or x.shape[1] != cols or (m_tokens is not None and m_tokens != x.shape[0]):
        raise ValueError(f"qkv must be [{'M' if m_tokens is None else m_tokens}, {cols}]")
    else:
        m_tokens = x.shape[0]
    for t, name in ((seq_start, "seq_start"), (key_len, "key_len")):
        if t is not None and (t.dtype != torch.int32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous 1-D CUDA int32 tensor")
    n_seq = seq_start.shape[0] - 1
    if n_seq < 0 or (key_len is not None and key_len.shape[0] != n_seq):
        raise ValueError("seq_start has n_seq + 1 entries, key_len n_seq")
    return m_tokens, n_kv, n_seq


def attention(qkv, x_scale: float, seq_start, max_len: int, n_heads: int, head_dim: int, *,
              n_kv_heads: Optional[int] = None, softmax_scale: Optional[float] = None, key_len=None,
              kind: int = EPI_I8, out_scale: float = 1.0, blocks=None, query_block: int = 64,
              x_layout: int = LAYOUT_ROWS, y_layout: int = LAYOUT_ROWS, m_tokens: Optional[int] = None, out=None,
              stream=None):
    """The attention core on a QKV linear's int8 output: codes of x_scale, [M,
    (n_heads + 2 n_kv_heads) * head_dim], query heads first, then keys, then values.

    Sequence s is tokens seq_start[s] .. seq_start[s+1]-1 (int32 on the device;
    max_len: the longest, which sizes the launch); key_len: valid keys of each,
    default all. softmax_scale: default 1 / sqrt(head_dim). blocks: lists of
    select_blocks with the same query_block, to attend to those keys only.
    Returns [M, n_heads * head_dim]: int8 codes of out_scale (EPI_I8, y_layout) or
    fp32 (EPI_F32). Tokens of no sequence are left as they are."""
    m, n_kv, n_seq = _attention_args(qkv, seq_start, max_len, n_heads, head_dim, n_kv_heads, key_len, x_layout,
                                     m_tokens)
    torch = _torch
    cols = n_heads * head_dim
    dt = _KIND_DTYPE.get(kind)
    shape = t16x32_shape(m, cols) if y_layout == LAYOUT_T16X32 else (m, cols)
    if out is None:
        out = _empty(shape, dt, qkv.device, stream)
    elif out.dtype != dt or tuple(out.shape) != shape or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out has the wrong dtype/shape or is not contiguous")
    lists, top_k = 0, 0
    if blocks is not None:
        if query_block < 1:
            raise ValueError("query_block must be >= 1")
        want = (n_seq, n_heads, -(-max_len // query_block))
        if blocks.dtype != torch.int32 or not blocks.is_cuda or not blocks.is_contiguous() or blocks.dim() != 4 or \
                tuple(blocks.shape[:3]) != want:
            raise ValueError(f"blocks must be a contiguous CUDA int32 tensor of shape {want} and a list each")
        lists, top_k = blocks.data_ptr(), blocks.shape[3]
    args = _ATTN_ARGS.pack(qkv.data_ptr(), m, seq_start.data_ptr(), 0 if key_len is None else key_len.data_ptr(), lists,
                           out.data_ptr(), n_seq, max_len, x_layout, n_heads, n_kv, head_dim, top_k, query_block, kind,
                           y_layout, x_scale, head_dim ** -0.5 if softmax_scale is None else softmax_scale, out_scale)
    st = load().attention_run(args, _stream_ptr(stream))
    if st != SL_OK:
        _check(st, "attention_run")
    return out


def select_blocks(qkv, seq_start, max_len: int, n_heads: int, head_dim: int, top_k: int, *,
                  n_kv_heads: Optional[int] = None, query_block: int = 64, key_len=None,
                  x_layout: int = LAYOUT_ROWS, m_tokens: Optional[int] = None, out=None, stream=None):
    """For every block of query_block queries and head, the top_k blocks of 64 keys
    by the product of the pooled queries and keys (whole numbers: exact; ties to
    the lowest block). Other arguments as attention's. Returns int32 [n_seq,
    n_heads, ceil(max_len / query_block), top_k], ascending, then -1."""
    m, n_kv, n_seq = _attention_args(qkv, seq_start, max_len, n_heads, head_dim, n_kv_heads, key_len, x_layout,
                                     m_tokens)
    torch = _torch
    if query_block < 1 or top_k < 1 or n_heads < 0 or max_len < 0:
        raise ValueError("query_block and top_k must be >= 1, n_heads and max_len >= 0")
    shape = (n_seq, n_heads, -(-max_len // query_block), top_k)
    if out is None:
        out = _empty(shape, torch.int32, qkv.device, stream)
    elif out.dtype != torch.int32 or tuple(out.shape) != shape or not out.is_contiguous() or not out.is_cuda:
        raise ValueError(f"out must be a contiguous CUDA int32 tensor of shape {shape}")
    if m == 0:  # (the call writes nothing)
        with torch.cuda.stream(stream):  # (None: the current one)
            return out.fill_(-1)
    args = _ATTN_ARGS.pack(qkv.data_ptr(), m, seq_start.data_ptr(), 0 if key_len is None else key_len.data_ptr(), 0, 0,
                           n_seq, max_len, x_layout, n_heads, n_kv, head_dim, top_k, query_block, EPI_F32, LAYOUT_ROWS,
                           1.0, 1.0, 1.0)
    lib, s = load(), _stream_ptr(stream)
    size = lib.attention_select_workspace(args)
    # from the memory of the stream that uses it, which is not handed on before that work is done
    if stream is None:
        work = torch.empty(size, dtype=torch.uint8, device=qkv.device)
    else:
        with torch.cuda.stream(stream):
            work = torch.empty(size, dtype=torch.uint8, device=qkv.device)
    st = lib.attention_select(args, out.data_ptr(), work.data_ptr(), size, s)
    if st != SL_OK:
        _check(st, "attention_select")
    return out


# --- a decoder's cache ----------------------------------------------------------

def cache_shape(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int):
    """Shape of a key-value cache: pages, keys and values, heads. Keys of a page and head are [page_size, head_dim],
    values, in the same shape's memory, [page_size / 16, head_dim, 16]."""
    return (n_pages, 2, n_kv_heads, page_size, head_dim)


def _cache_args(x, name, cache, page_table, seq_start, kv_len, stream):
    """Checks of what cache_append and cache_attention share; returns (n_seq, pages of a sequence, the cache's shape, the
    stream's number). The launch goes to the current device, so the tensors (and the stream) have to be there."""
    torch = _torch or _torch_once()
    dev, i32, shape, table = x.get_device(), torch.int32, cache.shape, page_table.shape
    if dev < 0 or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if cache.dtype is not torch.int8 or len(shape) != 5 or shape[1] != 2 or not cache.is_contiguous():
        raise ValueError("cache must be a contiguous int8 tensor of cache_shape()")
    if page_table.dtype is not i32 or len(table) != 2 or not page_table.is_contiguous():
        raise ValueError("page_table must be a contiguous int32 tensor [n_seq, pages]")
    n_seq, pages = table
    if seq_start.dtype is not i32 or kv_len.dtype is not i32 or kv_len.shape != (n_seq,) or \
            seq_start.shape != (n_seq + 1,) or not seq_start.is_contiguous() or not kv_len.is_contiguous():
        raise ValueError("seq_start and kv_len must be contiguous int32 tensors [n_seq + 1] and [n_seq], as page_table's")
    if not (cache.get_device() == page_table.get_device() == seq_start.get_device() == kv_len.get_device() == dev):
        raise ValueError(f"cache, page_table, seq_start and kv_len must be on {name}'s device")
    if torch._C._cuda_getDevice() != dev or (stream is not None and stream.device_index != dev):
        raise ValueError("the tensors' device must be the current one, and the stream's")
    return n_seq, pages, shape, _stream_ptr(stream)


def cache_append(x, cache, page_table, seq_start, kv_len, max_new: int, n_heads: int, *, x_scale: float = 1.0,
                 k_scale: float, v_scale: float, q_scale: Optional[float] = None, rope: int = ROPE_NONE, inv_freq=None,
                 rope_factor: float = 1.0, positions=None, x_layout: int = LAYOUT_ROWS, q_layout: int = LAYOUT_ROWS,
                 m_tokens: Optional[int] = None, out=None, stream=None):
    """A QKV linear's output, [M, (n_heads + 2 n_kv_heads) * head_dim] fp32 or int8 codes of x_scale in x_layout, into
    the pages of a cache (cache_shape; codes of k_scale and v_scale) and to query codes of q_scale, queries and keys
    rotated by position.

    Sequence s is tokens seq_start[s] .. seq_start[s+1]-1 (at most max_new, which sizes the launch), the last of its
    kv_len[s] cached ones; page_table [n_seq, pages] names its pages (-1: none, not stored). inv_freq: fp32, one a
    rotated pair (rope: ROPE_HALF pairs j with j + R / 2, ROPE_INTERLEAVED 2 j with 2 j + 1), angles position *
    inv_freq; positions: int32 [M], default a token's slot; rope_factor multiplies both parts. n_heads may be 0 (an
    encoder's keys and values). Returns the query codes [M, n_heads * head_dim] in q_layout, or None without q_scale.
    Tokens of no sequence are left as they are."""
    torch = _torch or _torch_once()
    n_seq, pages, (n_pages, _, n_kv, page_size, head_dim), s = _cache_args(x, "x", cache, page_table, seq_start, kv_len,
                                                                           stream)
    cols, have, dt = (n_heads + 2 * n_kv) * head_dim, x.shape, x.dtype
    x_type = ACT_F32 if dt is torch.float32 else ACT_I8
    if x_type == ACT_I8 and dt is not torch.int8:
        raise ValueError("x must be float32 or int8")
    if x_layout == LAYOUT_T16X32:
        if x_type == ACT_F32 or m_tokens is None:
            raise ValueError("LAYOUT_T16X32 input is int8, and needs m_tokens")
        if have != t16x32_shape(m_tokens, cols):
            raise ValueError(f"x must have shape {t16x32_shape(m_tokens, cols)}")
    elif len(have) != 2 or have[1] != cols or (m_tokens is not None and m_tokens != have[0]):
        raise ValueError(f"x must be [{'M' if m_tokens is None else m_tokens}, {cols}]")
    else:
        m_tokens = have[0]
    q = None
    if q_scale is not None:
        shape = t16x32_shape(m_tokens, n_heads * head_dim) if q_layout == LAYOUT_T16X32 else (m_tokens, n_heads * head_dim)
        if out is None:
            q = _empty(shape, torch.int8, x.device, stream)
        else:
            q = out
            if q.dtype is not torch.int8 or q.shape != shape or not q.is_contiguous() or q.device != x.device:
                raise ValueError(f"out must be a contiguous int8 tensor of shape {shape} on x's device")
    rope_dim = freq = at = 0
    if rope != ROPE_NONE:
        if inv_freq is None or inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or \
                not inv_freq.is_contiguous() or inv_freq.device != x.device:
            raise ValueError("inv_freq must be a contiguous 1-D float32 tensor on x's device")
        rope_dim, freq = 2 * inv_freq.shape[0], inv_freq.data_ptr()
        if positions is not None:
            if positions.dtype is not torch.int32 or positions.shape != (m_tokens,) or \
                    not positions.is_contiguous() or positions.device != x.device:
                raise ValueError("positions must be a contiguous int32 tensor [M] on x's device")
            at = positions.data_ptr()
    args = _APPEND_ARGS.pack(
        x.data_ptr(), m_tokens, seq_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), at, freq, cache.data_ptr(),
        0 if q is None else q.data_ptr(), n_seq, max_new, pages, n_pages, page_size, x_type, x_layout, n_heads,
        n_kv, head_dim, rope, rope_dim, q_layout, x_scale, rope_factor, 1.0 if q_scale is None else q_scale, k_scale, v_scale)
    st = load().cache_append(args, s)
    if st != SL_OK:
        _check(st, "cache_append")
    return q


def cache_attention(q, cache, page_table, seq_start, kv_len, max_new: int, max_len: int, n_heads: int, *, q_scale: float,
                    k_scale: float, v_scale: float, softmax_scale: Optional[float] = None, causal: bool = True,
                    kind: int = EPI_I8, out_scale: float = 1.0, q_cols: Optional[int] = None,
                    q_layout: int = LAYOUT_ROWS, y_layout: int = LAYOUT_ROWS, m_tokens: Optional[int] = None, out=None,
                    stream=None):
    """Attention of a call's tokens (query codes [M, n_heads * head_dim] of q_scale, or wider rows that begin with them:
    q_cols, in the block layout) over what their sequences have in the cache: one token a sequence, some, or prompts.

    Sequences as in cache_append; max_new and max_len, the largest of their tokens and of kv_len, size the launch (what is
    longer is still done whole; a bound far over the lengths, or a long prompt among many steps, takes longer). With causal a token sees the slots up to its own, else all kv_len[s] (an encoder's states). softmax_scale: default
    1 / sqrt(head_dim). Returns [M, n_heads * head_dim]: int8 codes of out_scale (EPI_I8, y_layout) or fp32 (EPI_F32); 0
    where nothing is seen. Tokens of no sequence are left as they are."""
    torch = _torch or _torch_once()
    n_seq, pages, (n_pages, _, n_kv, page_size, head_dim), s = _cache_args(q, "q", cache, page_table, seq_start, kv_len,
                                                                           stream)
    if q.dtype is not torch.int8:
        raise ValueError("q must be int8")
    cols, have = n_heads * head_dim, q.shape
    if q_layout == LAYOUT_T16X32:
        q_cols = cols if q_cols is None else q_cols
        if m_tokens is None:
            raise ValueError("m_tokens is required with LAYOUT_T16X32 input")
        if have != t16x32_shape(m_tokens, q_cols):
            raise ValueError(f"q must have shape {t16x32_shape(m_tokens, q_cols)}")
    elif len(have) != 2 or (m_tokens is not None and m_tokens != have[0]) or \
            (q_cols is not None and q_cols != have[1]) or have[1] < cols:
        raise ValueError(f"q must be [{'M' if m_tokens is None else m_tokens}, {cols} or more]")
    else:
        m_tokens, q_cols = have
    dt = _KIND_DTYPE.get(kind)
    shape = t16x32_shape(m_tokens, cols) if y_layout == LAYOUT_T16X32 else (m_tokens, cols)
    if out is None:  # (empty_like: 0.6 us less a call)
        out = torch.empty_like(q) if dt is torch.int8 and have == shape and stream is None else \
            _empty(shape, dt, q.device, stream)
    elif out.dtype is not dt or out.shape != shape or not out.is_contiguous() or out.device != q.device:
        raise ValueError("out has the wrong dtype/shape/device or is not contiguous")
    if softmax_scale is None:
        softmax_scale = head_dim ** -0.5 if head_dim else 1.0  # (no head: refused below)
    fields = (n_seq, max_new, max_len, pages, n_pages, page_size, q_layout, q_cols, n_heads, n_kv, head_dim,
              1 if causal else 0, kind, y_layout, q_scale, k_scale, v_scale, softmax_scale, out_scale)
    head = (q.data_ptr(), m_tokens, seq_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), cache.data_ptr(),
            out.data_ptr())
    lib, args = load(), _CACHE_ARGS.pack(*head, 0, 0, *fields)
    st = lib.cache_attention(args, s)  # (most calls need no workspace, and one that does is refused first)
    if st != SL_OK:
        size = lib.cache_attention_workspace(args)
        if size:
            # from the memory of the stream that uses it, which is not handed on before that work is done
            if stream is None:
                work = torch.empty(size, dtype=torch.uint8, device=q.device)
            else:
                with torch.cuda.stream(stream):
                    work = torch.empty(size, dtype=torch.uint8, device=q.device)
            args = _CACHE_ARGS.pack(*head, work.data_ptr(), size, *fields)
        st = lib.cache_attention(args, s)
    if st != SL_OK:
        _check(st, "cache_attention")
    return out
