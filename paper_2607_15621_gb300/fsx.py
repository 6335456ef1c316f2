"""Thin binding of libfsx.so (include/fsx.h): argument marshalling only, by ctypes, and for
the operators over a cache in pages by an extension module (csrc/calls.cpp).

Every step of the tick runs in the library's CUDA kernels; this module only
turns torch tensors / numpy arrays into pointers, sizes and a cudaStream_t.
Importing it fails loudly when the compiled library is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import Sequence

import numpy as np

from .synth import Dims

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "_lib", "libfsx.so")
CALLS_PATH = os.path.join(_PKG, "_lib", "_calls.so")

FSX_OK = 0
FSX_ERR_INVALID_ARG = 1
FSX_ERR_UNSUPPORTED = 2
FSX_ERR_OOM = 3
FSX_ERR_CUDA = 4
FSX_ERR_TIMEOUT = 5
FSX_ERR_DEVICE_ARG = 6
FSX_ERR_RANGE = 7
FSX_F32 = 0
FSX_BF16 = 1
FSX_F16 = 2
FSX_E4M3 = 3
FSX_ROTARY_HALVES = 0
FSX_ROTARY_ADJACENT = 1
FSX_SCHED_SERIAL = 0
FSX_SCHED_CONCURRENT = 1

KCLASS = {"qkv": 0, "attention": 1, "out_proj": 2, "gate_up": 3, "down": 4, "persistent": 5}


class FsxError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"fsx status {status}: {message}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("d_model", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("d_ff", ctypes.c_int), ("n_action", ctypes.c_int),
                ("n_frame", ctypes.c_int), ("n_waypoints", ctypes.c_int), ("max_batch", ctypes.c_int),
                ("max_total_cache_tokens", ctypes.c_longlong), ("cache_dtype", ctypes.c_int),
                ("frame_dtype", ctypes.c_int)]


_WEIGHT_FIELDS = ["act_emb", "pos_emb", "attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate",
                  "w_up", "w_down", "final_norm", "head_w", "head_b"]


class Weights(ctypes.Structure):
    _fields_ = [(name, ctypes.POINTER(ctypes.c_float)) for name in _WEIGHT_FIELDS]


_PAPER_WEIGHT_FIELDS = ["state_w1", "state_b1", "state_w2", "state_b2", "query_emb", "pos_emb", "attn_norm", "wq",
                        "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down", "final_norm", "head_w1", "head_b1",
                        "head_w2", "head_b2"]


class PaperWeights(ctypes.Structure):
    _fields_ = [(name, ctypes.POINTER(ctypes.c_float)) for name in _PAPER_WEIGHT_FIELDS]


class AppendConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("d_model", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("d_ff", ctypes.c_int), ("n_new", ctypes.c_int),
                ("max_batch", ctypes.c_int), ("max_cache_rows", ctypes.c_longlong), ("rope_base", ctypes.c_float)]


_APPEND_WEIGHT_FIELDS = ["attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down"]


class AppendWeights(ctypes.Structure):
    _fields_ = [(name, ctypes.POINTER(ctypes.c_float)) for name in _APPEND_WEIGHT_FIELDS]


class PagePlane(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("page_bytes", ctypes.c_longlong), ("segment_stride", ctypes.c_longlong),
                ("segments", ctypes.c_int)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2607_15621_gb300.build.build()")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64p = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_int64)
    vpp = ctypes.POINTER(ctypes.c_void_p)
    fp = ctypes.POINTER(ctypes.c_float)
    ll = ctypes.c_longlong
    sig = {
        "fsx_create": (i32, [ctypes.POINTER(Config), ctypes.POINTER(Weights), i32, ctypes.POINTER(vp)]),
        "fsx_tick": (i32, [vp, vpp, vpp, vp, i32, vp, vp, vp]),
        "fsx_tick_host": (i32, [vp, vpp, vpp, vp, i32, vp, vp, vp]),
        "fsx_tick_debug": (i32, [vp, vpp, vpp, vp, i32, vp, vp, vp, vp]),
        "fsx_tick_ranges": (i32, [vp, vpp, vpp, vp, vp, i32, vp, vp, vp]),
        "fsx_tick_ranges_debug": (i32, [vp, vpp, vpp, vp, vp, i32, vp, vp, vp, vp]),
        "fsx_get_status": (i32, [vp, vp]),
        "fsx_last_error": (ctypes.c_char_p, []),
        "fsx_destroy": (None, [vp]),
        "fsx_set_wait_limit": (i32, [vp, ctypes.c_ulonglong]),
        "fsx_weight_bytes": (ctypes.c_longlong, [vp]),
        "fsx_tick_launches": (i32, [vp, i32]),
        "fsx_set_kernel_timing": (i32, [vp, i32, i32]),
        "fsx_kernel_time": (i32, [vp, fp, ctypes.POINTER(ctypes.c_int)]),
        "fsx_attention_workspace_bytes": (ctypes.c_size_t, [i32, i32, i32, i32]),
        "fsx_attention": (i32, [vp, ctypes.c_longlong, vp, vp, ctypes.c_longlong, i32, i32, vp, vp, i32,
                                vp, i32, i32, i32, i32, vp, vp, vp, ctypes.c_size_t, vp]),
        "fsx_attention_noalloc": (i32, [vp, ctypes.c_longlong, vp, vp, ctypes.c_longlong, i32, i32, vp, vp,
                                        i32, vp, i32, i32, i32, i32, vp, vp, vp]),
        "fsx_attention_noalloc_status": (i32, [vp]),
        "fsx_paper_create": (i32, [ctypes.POINTER(Config), ctypes.POINTER(PaperWeights), i32, ctypes.POINTER(vp)]),
        "fsx_paper_tick": (i32, [vp, vpp, vpp, vp, i32, vp, vp, vp, vp]),
        "fsx_append_set_concurrent": (i32, [vp, i32]),
        "fsx_session_create": (i32, [vp, vp, vpp, vpp, i32, i32, ctypes.c_longlong, ctypes.c_longlong, i32, i32,
                                     ctypes.POINTER(vp)]),
        "fsx_session_append": (i32, [vp, vp, vp]),
        "fsx_session_tick": (i32, [vp, vp, vp, ctypes.POINTER(ctypes.c_longlong)]),
        "fsx_session_committed": (ctypes.c_longlong, [vp]),
        "fsx_session_reserved": (ctypes.c_longlong, [vp]),
        "fsx_session_tick_stream": (vp, [vp]),
        "fsx_session_append_stream": (vp, [vp]),
        "fsx_session_sync": (i32, [vp]),
        "fsx_session_destroy": (None, [vp]),
        "fsx_append_create": (i32, [ctypes.POINTER(AppendConfig), ctypes.POINTER(AppendWeights), i32,
                                    ctypes.POINTER(vp)]),
        "fsx_append": (i32, [vp, vpp, vpp, vp, vp, i32, vp, vp, vp]),
        "fsx_append_get_status": (i32, [vp, vp]),
        "fsx_append_weight_bytes": (ctypes.c_longlong, [vp]),
        "fsx_append_destroy": (None, [vp]),
        "fsx_cache_write_e4m3": (i32, [vp, vp, ll, i32, vp, ll, i32, i32, vp, vp, vp, vp, ll, vp, vp]),
        "fsx_cache_read_e4m3": (i32, [vp, vp, vp, vp, ll, vp, ll, i32, i32, vp, vp, ll, i32, vp, vp]),
        "fsx_prompt_attention": (i32, [vp, ll, vp, vp, ll, i32, vp, vp, i32, ll, ll, i32, i32, i32, i32, vp, vp, vp,
                                       vp]),
        "fsx_tree_attention_workspace_bytes": (ctypes.c_size_t, [i32, ll, i32, i32]),
        "fsx_tree_attention": (i32, [vp, ll, vp, vp, ll, i32, vp, vp, ll, vp, vp, vp, vp, i32, ll, vp, vp, i32, i32,
                                     i32, i32, vp, vp, vp, ctypes.c_size_t, vp, vp]),
        "fsx_rotary": (i32, [vp, ll, vp, vp, ll, i32, vp, i32, vp, vp, i32, ll, i32, i32, i32, vp, ll, vp, ll, vp, vp, vp, vp,
                             vp, i32, ll, vp, vp]),
        "fsx_paged_attention_workspace_bytes": (ctypes.c_size_t, [i32, i32, i32]),
        "fsx_paged_attention": (i32, [vp, ll, i32, vp, vp, vp, vp, i32, ll, i32, vp, i32, vp, i32, vp, i32, i32, i32, i32, vp, vp,
                                      vp, ctypes.c_size_t, vp, vp]),
        "fsx_page_bounds": (i32, [vp, vp, i32, ll, i32, vp, i32, vp, vp, i32, i32, i32, vp, vp, vp, vp]),
        "fsx_page_select": (i32, [vp, ll, i32, vp, vp, ll, i32, vp, i32, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]),
        "fsx_pages_step": (i32, [vp, vp, vp, i32, vp, vp, i32, ll, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]),
        "fsx_pages_compact": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp]),
        "fsx_pages_copy": (i32, [vp, i32, i32, vp, vp, i32, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = None


def lib():
    global _lib
    if _lib is None:
        _lib = _load()
    return _lib


def declared_symbols() -> list[str]:
    return ["fsx_create", "fsx_tick", "fsx_tick_host", "fsx_tick_debug", "fsx_tick_ranges", "fsx_tick_ranges_debug",
            "fsx_get_status", "fsx_last_error",
            "fsx_destroy", "fsx_weight_bytes", "fsx_tick_launches", "fsx_set_kernel_timing",
            "fsx_kernel_time", "fsx_attention_workspace_bytes", "fsx_attention", "fsx_attention_noalloc",
            "fsx_attention_noalloc_status", "fsx_paper_create", "fsx_paper_tick", "fsx_append_create", "fsx_append",
            "fsx_append_get_status", "fsx_append_weight_bytes", "fsx_append_destroy", "fsx_append_set_concurrent",
            "fsx_session_create", "fsx_session_append", "fsx_session_tick", "fsx_session_committed",
            "fsx_session_reserved", "fsx_session_tick_stream", "fsx_session_append_stream", "fsx_session_sync",
            "fsx_session_destroy", "fsx_set_wait_limit", "fsx_cache_write_e4m3", "fsx_cache_read_e4m3",
            "fsx_prompt_attention", "fsx_tree_attention_workspace_bytes", "fsx_tree_attention", "fsx_rotary",
            "fsx_paged_attention_workspace_bytes", "fsx_paged_attention", "fsx_page_bounds", "fsx_page_select",
            "fsx_pages_step", "fsx_pages_compact", "fsx_pages_copy"]


def last_error() -> str:
    return lib().fsx_last_error().decode()


def check(status: int):
    if status != FSX_OK:
        raise FsxError(status, last_error())


def _ptr(t) -> int:
    """Device or host address of a torch tensor / numpy array (None -> 0)."""
    if t is None:
        return 0
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:  # torch.cuda.current_stream().cuda_stream without the Stream object: 3.0 -> 0.4 us
        # a call, and of Eq. 1 for one vehicle, back to back, 24-26 -> 20.5 us
        import torch
        torch.cuda.init()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ptr_array(tensors: Sequence) -> ctypes.Array:
    arr = (ctypes.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = _ptr(t)
    return arr


def make_config(dims: Dims, max_batch: int, max_total_cache_tokens: int, cache_dtype: str = "bf16",
                frame_dtype: str = "bf16") -> Config:
    code = {"fp32": FSX_F32, "bf16": FSX_BF16}
    return Config(dims.n_layers, dims.d_model, dims.n_heads, dims.head_dim, dims.d_ff, dims.n_action,
                  dims.n_frame, dims.n_waypoints, max_batch, max_total_cache_tokens,
                  code[cache_dtype], code[frame_dtype])


def make_weights(weights: dict):
    """ctypes struct of host fp32 pointers plus the contiguous arrays it points to."""
    keep = {k: np.ascontiguousarray(weights[k], dtype=np.float32) for k in _WEIGHT_FIELDS}
    st = Weights(*[keep[k].ctypes.data_as(ctypes.POINTER(ctypes.c_float)) for k in _WEIGHT_FIELDS])
    return st, keep


class Expert:
    """Owns one fsx handle (weights uploaded at construction)."""

    def __init__(self, dims: Dims, weights: dict, max_batch: int, max_total_cache_tokens: int,
                 cache_dtype: str = "bf16", frame_dtype: str = "bf16", device: int = 0):
        self.dims = dims
        self.cfg = make_config(dims, max_batch, max_total_cache_tokens, cache_dtype, frame_dtype)
        wst, keep = make_weights(weights)
        h = ctypes.c_void_p()
        check(lib().fsx_create(ctypes.byref(self.cfg), ctypes.byref(wst), device, ctypes.byref(h)))
        self.h = h
        del keep

    def close(self):
        if getattr(self, "h", None) and self.h.value:
            lib().fsx_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def tick(self, k_layers, v_layers, offsets, frames, out, stream=None, starts=None):
        """One tick; with `starts`, vehicle b reads rows starts[b] .. starts[b] + L_b - 1."""
        B = int(frames.shape[0])
        if starts is None:
            check(lib().fsx_tick(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(offsets), B,
                                 _ptr(frames), _ptr(out), _stream(stream)))
        else:
            check(lib().fsx_tick_ranges(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(starts),
                                        _ptr(offsets), B, _ptr(frames), _ptr(out), _stream(stream)))
        return out

    def tick_host(self, k_layers, v_layers, offsets_host: np.ndarray, frames_host, out_host: np.ndarray,
                  stream=None):
        B = int(frames_host.shape[0])
        check(lib().fsx_tick_host(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(offsets_host), B,
                                  _ptr(frames_host), _ptr(out_host), _stream(stream)))
        return out_host

    def tick_debug(self, k_layers, v_layers, offsets, frames, out, attn_out, stream=None, starts=None):
        B = int(frames.shape[0])
        if starts is None:
            check(lib().fsx_tick_debug(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(offsets), B,
                                       _ptr(frames), _ptr(out), _ptr(attn_out), _stream(stream)))
        else:
            check(lib().fsx_tick_ranges_debug(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(starts),
                                              _ptr(offsets), B, _ptr(frames), _ptr(out), _ptr(attn_out),
                                              _stream(stream)))
        return out, attn_out

    def status(self, stream=None) -> int:
        return lib().fsx_get_status(self.h, _stream(stream))

    def weight_bytes(self) -> int:
        return int(lib().fsx_weight_bytes(self.h))

    def set_wait_limit(self, ns: int):
        """Test hook: limit of the single-launch tick's device-wide waits (0 = the default 1 s)."""
        check(lib().fsx_set_wait_limit(self.h, ns))

    def launches(self, B: int) -> int:
        return int(lib().fsx_tick_launches(self.h, B))

    def set_kernel_timing(self, enable: bool, kclass: str = "qkv"):
        check(lib().fsx_set_kernel_timing(self.h, int(enable), KCLASS[kclass]))

    def kernel_time(self):
        ms = ctypes.c_float()
        n = ctypes.c_int()
        check(lib().fsx_kernel_time(self.h, ctypes.byref(ms), ctypes.byref(n)))
        return float(ms.value), int(n.value)


class PaperExpert(Expert):
    """A tick handle of the paper's ten-token layout (fsx_paper_create / fsx_paper_tick):
    state token, four visual tokens, five waypoint queries and a two-layer head over the
    same layer stack. Argument marshalling only."""

    def __init__(self, dims: Dims, weights: dict, max_batch: int, max_total_cache_tokens: int,
                 cache_dtype: str = "bf16", visual_dtype: str = "bf16", device: int = 0):
        self.dims = dims
        self.cfg = make_config(dims, max_batch, max_total_cache_tokens, cache_dtype, visual_dtype)
        keep = {k: np.ascontiguousarray(weights[k], dtype=np.float32) for k in _PAPER_WEIGHT_FIELDS}
        wst = PaperWeights(*[keep[k].ctypes.data_as(ctypes.POINTER(ctypes.c_float)) for k in _PAPER_WEIGHT_FIELDS])
        h = ctypes.c_void_p()
        check(lib().fsx_paper_create(ctypes.byref(self.cfg), ctypes.byref(wst), device, ctypes.byref(h)))
        self.h = h
        del keep

    def paper_tick(self, k_layers, v_layers, offsets, visual, state, out, stream=None):
        B = int(visual.shape[0])
        check(lib().fsx_paper_tick(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(offsets), B,
                                   _ptr(visual), _ptr(state), _ptr(out), _stream(stream)))
        return out


def attention_workspace_bytes(B: int, n_heads: int, n_q: int, n_splits: int) -> int:
    return int(lib().fsx_attention_workspace_bytes(B, n_heads, n_q, n_splits))


def attention(q, q_stride, k_own, v_own, own_stride, n_q, n_own, k_cache, v_cache, cache_dtype, offsets, B,
              n_heads, n_splits, out, lse, workspace, stream=None):
    """Eq. 1 alone through the C ABI (fp16 tensors, int64 offsets, caller scratch)."""
    code = {"fp32": FSX_F32, "bf16": FSX_BF16}[cache_dtype]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    check(lib().fsx_attention(_ptr(q), q_stride, _ptr(k_own), _ptr(v_own), own_stride, n_q, n_own,
                              _ptr(k_cache), _ptr(v_cache), code, _ptr(offsets), B, n_heads, 128, n_splits,
                              _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)))
    return out


def attention_noalloc(q, q_stride, k_own, v_own, own_stride, n_q, n_own, k_cache, v_cache, cache_dtype, offsets,
                      B, n_heads, n_splits, out, lse, stream=None):
    """fsx_attention_noalloc through the C ABI: same results as attention(), with the
    library's static scratch instead of a caller buffer (nothing is allocated)."""
    code = {"fp32": FSX_F32, "bf16": FSX_BF16}[cache_dtype]
    check(lib().fsx_attention_noalloc(_ptr(q), q_stride, _ptr(k_own), _ptr(v_own), own_stride, n_q, n_own,
                                      _ptr(k_cache), _ptr(v_cache), code, _ptr(offsets), B, n_heads, 128,
                                      n_splits, _ptr(out), _ptr(lse), _stream(stream)))
    return out


def attention_noalloc_status(stream=None) -> int:
    """fsx_attention_noalloc_status: synchronises the stream, returns and clears the
    device status word of the static scratch (FSX_OK, FSX_ERR_DEVICE_ARG or FSX_ERR_TIMEOUT)."""
    return int(lib().fsx_attention_noalloc_status(_stream(stream)))


# What the checks below ask for. A call of 10 to 20 us on the GPU waits for its caller: the conditions are one expression
# of cheap attributes (12 to 23 us a call with a helper for each), and only a refusal looks for its reason.
_CODES: dict = {}  # torch dtype -> fsx_dtype; e4m3 caches may be held as bytes
_I64 = _F32 = _raw_stream = _device = None


def _codes() -> dict:
    global _I64, _F32, _raw_stream, _device
    if not _CODES:
        import torch
        _I64, _F32 = torch.int64, torch.float32
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # of tensors on the GPU: CUDA is at work
        _device = getattr(torch._C, "_cuda_getDevice", None)
        _CODES.update({torch.float32: FSX_F32, torch.bfloat16: FSX_BF16, torch.float16: FSX_F16,
                       torch.float8_e4m3fn: FSX_E4M3, torch.uint8: FSX_E4M3})
    return _CODES


def _refuse(what: str, **tensors):
    """Raises for tensors that do not go together: `what` is asked for."""
    given = ", ".join(f"{n} {'None' if t is None else f'{tuple(t.shape)} {t.dtype} stride {t.stride()}'}"
                      for n, t in tensors.items())
    raise FsxError(FSX_ERR_INVALID_ARG, f"{what}; given: {given}")


def _rows(t, stride) -> bool:
    """[rows, heads, head_dim] whose rows are contiguous."""
    return stride[2] == 1 and (stride[1] == t.shape[2] or t.shape[1] == 1)


def _pitch(t, stride) -> int:
    return stride[0] if t.shape[0] > 1 else max(stride[0], t.shape[1] * t.shape[2])


def _alike(v, k) -> bool:
    """Rows as far apart in both, where the strides of an axis of one entry say nothing."""
    return _rows(v, v.stride()) and (v.shape[0] < 2 or v.stride(0) == k.stride(0))


def _cache8_call(k, v, rows, k_cache, v_cache, k_scale, v_scale):
    codes = _CODES or _codes()
    shape, stride, cs, ss, dtype, held = k.shape, k.stride(), k_cache.shape, k_scale.shape, k.dtype, k_cache.dtype
    good = (len(shape) == 3 and len(cs) == 3 and len(ss) == 2 and v.shape == shape and
            (v.stride() == stride or _alike(v, k)) and v.dtype is dtype and dtype in codes and
            stride[2] == 1 and (stride[1] == shape[2] or shape[1] == 1) and cs[1] == shape[1] and cs[2] == shape[2] and
            v_cache.shape == cs and v_cache.dtype is held and codes.get(held) == FSX_E4M3 and
            k_cache.is_contiguous() and v_cache.is_contiguous() and
            k_scale.dtype is _F32 and v_scale.dtype is _F32 and ss[0] == cs[1] and ss[1] == cs[0] and
            v_scale.shape == ss and k_scale.is_contiguous() and v_scale.is_contiguous() and
            (rows is None or (rows.dtype is _I64 and rows.shape == shape[:1] and rows.is_contiguous())))
    if not good:
        _refuse("rows k, v [n, kv heads, 128] of one shape, dtype and stride, 8-bit caches [rows, kv heads, 128], scales "
                "fp32 [kv heads, rows], row numbers int64 [n]", k=k, v=v, rows=rows, k_cache=k_cache, v_cache=v_cache,
                k_scale=k_scale, v_scale=v_scale)
    return codes[dtype], shape, stride[0] if shape[0] > 1 else _pitch(k, stride), cs[0]


def cache_write(k, v, rows, k_cache, v_cache, k_scale, v_scale, status, stream=None):
    """fsx_cache_write_e4m3: rows k, v [n, kv heads, 128] into cache rows `rows` (int64 [n], distinct; None: 0 .. n - 1)."""
    code, shape, pitch, m = _cache8_call(k, v, rows, k_cache, v_cache, k_scale, v_scale)
    on = _raw_stream(_device()) if stream is None else _stream(stream)
    error = (_lib or lib()).fsx_cache_write_e4m3(
        k.data_ptr(), v.data_ptr(), pitch, code, None if rows is None else rows.data_ptr(), shape[0], shape[1], shape[2],
        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), m, status.data_ptr(), on)
    if error:
        check(error)


def cache_read(k_cache, v_cache, k_scale, v_scale, rows, k, v, status, stream=None):
    """fsx_cache_read_e4m3: cache rows `rows` (int64 [n]; None: 0 .. n - 1) into k, v [n, kv heads, 128]."""
    code, shape, pitch, m = _cache8_call(k, v, rows, k_cache, v_cache, k_scale, v_scale)
    on = _raw_stream(_device()) if stream is None else _stream(stream)
    error = (_lib or lib()).fsx_cache_read_e4m3(
        k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), m,
        None if rows is None else rows.data_ptr(), shape[0], shape[1], shape[2], k.data_ptr(), v.data_ptr(), pitch, code,
        status.data_ptr(), on)
    if error:
        check(error)
    return k, v


def prompt_attention(q, k, v, q_offsets, kv_offsets, out, status, lse=None, causal=True, stream=None):
    """fsx_prompt_attention: packed q [rows, heads, 128], k and v [rows, kv heads, 128], int64 offsets [B + 1]."""
    codes = _CODES or _codes()
    dtype, qs, ks, q_shape, k_shape = q.dtype, q.stride(), k.stride(), q.shape, k.shape
    good = (len(q_shape) == 3 and len(k_shape) == 3 and k.dtype is dtype and v.dtype is dtype and out.dtype is dtype and
            v.shape == k_shape and (v.stride() == ks or _alike(v, k)) and out.shape == q_shape and out.is_contiguous() and
            q_shape[2] == k_shape[2] and _rows(q, qs) and _rows(k, ks) and q_offsets.dtype is _I64 and
            kv_offsets.dtype is _I64 and q_offsets.shape == kv_offsets.shape and q_offsets.dim() == 1 and
            q_offsets.is_contiguous() and kv_offsets.is_contiguous() and dtype in codes and
            (lse is None or (lse.dtype is _F32 and lse.shape == (q_shape[1], q_shape[0]) and lse.is_contiguous())))
    if not good:
        _refuse("q, out [rows, heads, 128], k, v [rows, kv heads, 128] of one dtype, k and v of one stride, out contiguous, "
                "offsets int64 [B + 1], lse fp32 [heads, rows]", q=q, k=k, v=v, q_offsets=q_offsets,
                kv_offsets=kv_offsets, out=out, lse=lse)
    on = _raw_stream(_device()) if stream is None else _stream(stream)
    error = (_lib or lib()).fsx_prompt_attention(
        q.data_ptr(), _pitch(q, qs), k.data_ptr(), v.data_ptr(), _pitch(k, ks), codes[dtype], q_offsets.data_ptr(),
        kv_offsets.data_ptr(), q_offsets.shape[0] - 1, q_shape[0], k_shape[0], q_shape[1], k_shape[1], q_shape[2],
        1 if causal else 0, out.data_ptr(), None if lse is None else lse.data_ptr(), status.data_ptr(), on)
    if error:
        check(error)
    return out


def tree_attention_workspace_bytes(B: int, new_rows: int, n_heads: int, n_kv_heads: int) -> int:
    return int(lib().fsx_tree_attention_workspace_bytes(B, new_rows, n_heads, n_kv_heads))


def tree_attention(q, k_new, v_new, new_offsets, mask, k_cache, v_cache, offsets, out, status, workspace, k_scale=None,
                   v_scale=None, starts=None, lse=None, stream=None):
    """fsx_tree_attention: the new tokens' q [rows, heads, 128], k_new and v_new [rows, kv heads, 128], mask int64
    [rows], over caches [rows, kv heads, 128] of q's dtype or e4m3 (then with scales [kv heads, rows])."""
    codes = _CODES or _codes()
    dtype, held, qs, ks, q_shape, k_shape, cs = (q.dtype, k_cache.dtype, q.stride(), k_new.stride(), q.shape, k_new.shape,
                                                 k_cache.shape)
    code, n_shape = codes.get(held), new_offsets.shape
    good = (len(q_shape) == 3 and len(k_shape) == 3 and len(cs) == 3 and len(n_shape) == 1 and dtype in codes and
            k_new.dtype is dtype and v_new.dtype is dtype and out.dtype is dtype and v_new.shape == k_shape and
            (v_new.stride() == ks or _alike(v_new, k_new)) and out.shape == q_shape and out.is_contiguous() and
            q_shape[0] == k_shape[0] and q_shape[2] == k_shape[2] and qs[2] == 1 and
            (qs[1] == q_shape[2] or q_shape[1] == 1) and ks[2] == 1 and (ks[1] == k_shape[2] or k_shape[1] == 1) and
            new_offsets.dtype is _I64 and offsets.dtype is _I64 and offsets.shape == n_shape and
            new_offsets.is_contiguous() and offsets.is_contiguous() and mask.dtype is _I64 and
            mask.shape == q_shape[:1] and mask.is_contiguous() and code is not None and v_cache.dtype is held and
            v_cache.shape == cs and cs[1] == k_shape[1] and cs[2] == k_shape[2] and k_cache.is_contiguous() and
            v_cache.is_contiguous() and
            (code != FSX_E4M3 or (k_scale is not None and v_scale is not None and k_scale.dtype is _F32 and
                                  v_scale.dtype is _F32 and k_scale.shape == (cs[1], cs[0]) and
                                  v_scale.shape == (cs[1], cs[0]) and k_scale.is_contiguous() and
                                  v_scale.is_contiguous())) and
            (starts is None or (starts.dtype is _I64 and starts.is_contiguous() and starts.dim() == 1 and
                                starts.shape[0] == n_shape[0] - 1)) and
            (lse is None or (lse.dtype is _F32 and lse.shape == (q_shape[1], q_shape[0]) and lse.is_contiguous())))
    if not good:
        _refuse("q, out [rows, heads, 128], k_new, v_new [rows, kv heads, 128] of one dtype, k_new and v_new of one stride, out "
                "contiguous, offsets int64 [B + 1], mask int64 [rows], caches [rows, kv heads, 128] of that dtype or e4m3 "
                "with scales fp32 [kv heads, rows], starts int64 [B], lse fp32 [heads, rows]", q=q, k_new=k_new,
                v_new=v_new, new_offsets=new_offsets, mask=mask, k_cache=k_cache, v_cache=v_cache, offsets=offsets,
                out=out, k_scale=k_scale, v_scale=v_scale, starts=starts, lse=lse)
    eight = code == FSX_E4M3
    on = _raw_stream(_device()) if stream is None else _stream(stream)
    error = (_lib or lib()).fsx_tree_attention(
        q.data_ptr(), _pitch(q, qs), k_new.data_ptr(), v_new.data_ptr(), _pitch(k_new, ks), codes[dtype],
        new_offsets.data_ptr(), mask.data_ptr(), q_shape[0], k_cache.data_ptr(), v_cache.data_ptr(),
        k_scale.data_ptr() if eight else None, v_scale.data_ptr() if eight else None, code, cs[0],
        None if starts is None else starts.data_ptr(), offsets.data_ptr(), n_shape[0] - 1, q_shape[1], k_shape[1],
        q_shape[2], out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), status.data_ptr(), on)
    if error:
        check(error)
    return out


class RotaryPairs:
    """Axis and rate (radians a position) of the 64 pairs of a head, and how they lie in it; see rotary_pairs()."""

    def __init__(self, axis: Sequence[int], rate: Sequence[float], adjacent: bool = False):
        if len(axis) != 64 or len(rate) != 64:
            raise FsxError(FSX_ERR_INVALID_ARG, f"64 axes and rates are asked for; given: {len(axis)} and {len(rate)}")
        self.axis, self.rate = (ctypes.c_int * 64)(*axis), (ctypes.c_double * 64)(*rate)
        self.axis_at, self.rate_at = ctypes.addressof(self.axis), ctypes.addressof(self.rate)
        self.n_axes = max(axis) + 1
        self.layout = FSX_ROTARY_ADJACENT if adjacent else FSX_ROTARY_HALVES


def rotary_pairs(sections: Sequence[int] = (64,), base: float = 10000.0, per_axis: bool = False,
                 adjacent: bool = False) -> RotaryPairs:
    """The pairs in sections, one axis after another: pair j turns by base^(-j / 64) a position, or, `per_axis`, the i-th of an
    axis' n pairs by base^(-i / n). Pair j is dims (j, j + 64), or (2 j, 2 j + 1) if `adjacent`."""
    if sum(sections) != 64 or min(sections) < 0:
        raise FsxError(FSX_ERR_INVALID_ARG, f"sections that add up to 64 pairs are asked for; given: {tuple(sections)}")
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    rate = [base ** -(i / n if per_axis else j / 64)
            for j, (i, n) in enumerate((i, n) for n in sections for i in range(n))]
    return RotaryPairs(axis, rate, adjacent)


# The operators over a cache in pages are called through an extension module (csrc/calls.cpp), which reads the tensors and checks
# that they go together; -1: they do not.
_calls = _where = None


def _native():
    """The extension's functions, and what gives the current device (-1 on a machine without a GPU)."""
    global _calls, _where
    if _calls is None:
        import importlib.util
        import torch
        lib()
        if not os.path.exists(CALLS_PATH):
            from .build import calls_lacks
            lacks = calls_lacks()
            raise RuntimeError(f"{CALLS_PATH} is missing: build it with paper_2607_15621_gb300.build.build()"
                               + (f" (not here: {lacks})" if lacks else ""))
        spec = importlib.util.spec_from_file_location("_calls", CALLS_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind(LIB_PATH)
        _codes()
        if torch.cuda.is_available():
            torch.cuda.init()
            _where = torch._C._cuda_getDevice
        else:
            _where = lambda: -1
        _calls = module
    return _calls


def _refused(error: int, what: str, **tensors):
    if error > 0:
        check(error)
    _refuse(what + ", all on the current device", **tensors)


def rotary(q, k, positions, pairs: RotaryPairs, status, q_out=None, k_out=None, v=None, rows=None, k_cache=None, v_cache=None,
           k_scale=None, v_scale=None, stream=None):
    """fsx_rotary: q [n, heads, 128] into q_out, k [n, kv heads, 128] into k_out (each may be its input; q or k may be None), by
    positions int64 [axes, n]; with caches [rows, kv heads, 128] of their dtype or e4m3 (then with scales [kv heads, rows])
    the rotated keys and v into cache rows `rows` (int64 [n], distinct; None: 0 .. n - 1)."""
    call = _calls or _native()
    device = _where()
    error = call.rotary(q, k, positions, pairs.axis_at, pairs.rate_at, pairs.n_axes, pairs.layout, status, q_out, k_out, v, rows, k_cache,
                        v_cache, k_scale, v_scale, device, _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "q, q_out [n, heads, 128], k, k_out, v [n, kv heads, 128] of one dtype, k and v of one stride, positions int64 "
                 "[axes, n], rows int64 [n], caches [rows, kv heads, 128] of that dtype or e4m3 with scales fp32 [kv heads, rows]",
                 q=q, k=k, v=v, positions=positions, q_out=q_out, k_out=k_out, rows=rows, k_cache=k_cache, v_cache=v_cache,
                 k_scale=k_scale, v_scale=v_scale)


def paged_attention_workspace_bytes(B: int, n_heads: int, n_kv_heads: int) -> int:
    return int(lib().fsx_paged_attention_workspace_bytes(B, n_heads, n_kv_heads))


def paged_attention(q, k_cache, v_cache, table, lengths, page_rows: int, out, status, workspace, k_scale=None, v_scale=None,
                    picked=None, lse=None, stream=None):
    """fsx_paged_attention: one token a request, q [B, heads, 128], over caches [rows, kv heads, 128] of q's dtype or e4m3
    (then with scales [kv heads, rows]) in pages of page_rows rows: table int32 [B, width], lengths int64 [B]; over all pages or
    those of `picked`, int32 [B, kv heads, n]."""
    call = _calls or _native()
    device = _where()
    error = call.paged_attention(q, k_cache, v_cache, table, lengths, page_rows, out, status, workspace, k_scale, v_scale, picked, lse,
                                 device, _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "q, out [B, heads, 128] of one dtype, out contiguous, caches [rows, kv heads, 128] of that dtype or e4m3 with "
                 "scales fp32 [kv heads, rows], table int32 [B, width], lengths int64 [B], picked int32 [B, kv heads, n], lse fp32 "
                 "[heads, B]", q=q, k_cache=k_cache, v_cache=v_cache, table=table, lengths=lengths, out=out, k_scale=k_scale,
                 v_scale=v_scale, picked=picked, lse=lse)
    return out


def page_bounds(k_cache, table, lengths, page_rows: int, bounds, bound_scale, status, k_scale=None, start=None, stream=None):
    """fsx_page_bounds: least and largest keys of the requests' pages (from row start int64 [B] on) into bounds int8
    [pages, kv heads, 2, 128] and bound_scale fp32 [kv heads, pages]."""
    call = _calls or _native()
    device = _where()
    error = call.page_bounds(k_cache, table, lengths, page_rows, bounds, bound_scale, status, k_scale, start, device,
                             _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "a cache [rows, kv heads, 128] (e4m3: with scales fp32 [kv heads, rows]), table int32 [B, width], lengths and "
                 "start int64 [B], bounds int8 [pages, kv heads, 2, 128], bound_scale fp32 [kv heads, pages]", k_cache=k_cache,
                 table=table, lengths=lengths, bounds=bounds, bound_scale=bound_scale, k_scale=k_scale, start=start)


def page_select(q, bounds, bound_scale, table, lengths, page_rows: int, picked, status, first: int = 1, last: int = 1, stream=None):
    """fsx_page_select: the pages that q [B, heads, 128] attends to into picked int32 [B, kv heads, n]: the request's `first` first
    and `last` last ones and those of the highest scores."""
    call = _calls or _native()
    device = _where()
    error = call.page_select(q, bounds, bound_scale, table, lengths, page_rows, picked, status, first, last, device,
                             _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "q [B, heads, 128], bounds int8 [pages, kv heads, 2, 128], bound_scale fp32 [kv heads, pages], table int32 "
                 "[B, width], lengths int64 [B], picked int32 [B, kv heads, n]", q=q, bounds=bounds, bound_scale=bound_scale,
                 table=table, lengths=lengths, picked=picked)
    return picked


def pages_step(table, lengths, refs, new_offsets, page_rows: int, table_out, lengths_out, refs_out, rows, pairs, n_pairs, status,
               source=None, stream=None):
    """fsx_pages_step: the state table int32 [B_in, width], lengths int64 [B_in], refs int32 [pages] into table_out, lengths_out,
    refs_out, where request i takes on request source[i] (int32 [B]; None: itself) and grows by the rows of new_offsets (int64
    [B + 1]); rows int64 [new rows], pairs int32 [B, 2] and n_pairs int32 [1] for cache_write and pages_copy."""
    call = _calls or _native()
    device = _where()
    error = call.pages_step(table, lengths, refs, new_offsets, page_rows, table_out, lengths_out, refs_out, rows, pairs, n_pairs, status,
                            source, device, _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "table int32 [B_in, width], lengths int64 [B_in], refs int32 [pages], new_offsets int64 [B + 1], the same of B "
                 "requests, rows int64 [new rows], pairs int32 [B, 2], n_pairs int32 [1], source int32 [B]", table=table,
                 lengths=lengths, refs=refs, new_offsets=new_offsets, table_out=table_out, lengths_out=lengths_out,
                 refs_out=refs_out, rows=rows, pairs=pairs, n_pairs=n_pairs, source=source)


def pages_compact(table, lengths, refs, page_rows: int, table_out, refs_out, pairs, n_pairs, status, stream=None):
    """fsx_pages_compact: pages in use to the front; pairs int32 [pages / 2 or more, 2], n_pairs int32 [1] for pages_copy."""
    call = _calls or _native()
    device = _where()
    error = call.pages_compact(table, lengths, refs, page_rows, table_out, refs_out, pairs, n_pairs, status, device,
                               _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "table, table_out int32 [B, width], lengths int64 [B], refs, refs_out int32 [pages], pairs int32 [pages / 2 or "
                 "more, 2], n_pairs int32 [1]", table=table, lengths=lengths, refs=refs, table_out=table_out, refs_out=refs_out,
                 pairs=pairs, n_pairs=n_pairs)


class PagePlanes:
    """What a copy of pages moves; see page_planes(). Keeps the tensors."""

    def __init__(self, planes: Sequence, n_pages: int, keep: Sequence):
        self.array, self.n, self.n_pages, self._keep = (PagePlane * len(planes))(*planes), len(planes), n_pages, list(keep)
        self.at, self.device = ctypes.addressof(self.array), self._keep[0].get_device()  # -1: not on a GPU


def page_planes(page_rows: int, caches: Sequence = (), scales: Sequence = (), bounds: Sequence = (),
                bound_scales: Sequence = ()) -> PagePlanes:
    """The planes of caches [rows, kv heads, 128], scales [kv heads, rows], bounds [pages, kv heads, 2, 128] and bound scales
    [kv heads, pages], of all layers, keys and values: made once, used by every pages_copy."""
    groups = ((caches, 3, 0, page_rows), (scales, 2, 1, page_rows), (bounds, 4, 0, 1), (bound_scales, 2, 1, 1))
    each = [(t, t.shape[axis] // rows if t.dim() == dim and rows > 0 and t.numel() > 0 and t.shape[axis] % rows == 0 else 0)
            for group, dim, axis, rows in groups for t in group]
    if len({n for _, n in each}) != 1 or each[0][1] < 1 or len({t.device for t, _ in each}) != 1 or not all(t.is_contiguous() for t, _ in each):
        _refuse("caches [rows, kv heads, 128], scales [kv heads, rows], bounds [pages, kv heads, 2, 128], bound scales [kv heads, pages], "
                "contiguous, of as many whole pages each, on one device", **{f"planes[{i}]": t for i, (t, _) in enumerate(each)})
    n_pages, planes = each[0][1], []
    for group, by_row in ((caches, True), (scales, False), (bounds, True), (bound_scales, False)):
        for t in group:
            size = t.numel() * t.element_size()
            if by_row:
                planes.append(PagePlane(t.data_ptr(), size // t.shape[0] * (t.shape[0] // n_pages), 0, 1))
            else:
                planes.append(PagePlane(t.data_ptr(), t.element_size() * (t.shape[1] // n_pages), t.stride(0) * t.element_size(), t.shape[0]))
    return PagePlanes(planes, n_pages, [t for t, _ in each])


def pages_copy(planes: PagePlanes, pairs, n_pairs, status, stream=None):
    """fsx_pages_copy: page pairs[i, 0] to page pairs[i, 1] in every plane, for the first n_pairs of them."""
    call = _calls or _native()
    device = _where()
    error = -1 if planes.device != device else call.pages_copy(
        planes.at, planes.n, planes.n_pages, pairs, n_pairs, status, device, _raw_stream(device) if stream is None else _stream(stream))
    if error:
        _refused(error, "planes, pairs int32 [n, 2] and n_pairs int32 [1]", pairs=pairs, n_pairs=n_pairs)


class Append:
    """Owns one fsx_append handle: the backbone's incremental cache append
    (weights uploaded at construction). Argument marshalling only."""

    def __init__(self, dims, weights: dict, max_batch: int, max_cache_rows: int, device: int = 0):
        self.dims = dims
        self.cfg = AppendConfig(dims.n_layers, dims.d_model, dims.n_heads, dims.head_dim, dims.d_ff, dims.n_new,
                                max_batch, max_cache_rows, float(dims.rope_base))
        keep = {k: np.ascontiguousarray(weights[k], dtype=np.float32) for k in _APPEND_WEIGHT_FIELDS}
        wst = AppendWeights(*[keep[k].ctypes.data_as(ctypes.POINTER(ctypes.c_float)) for k in _APPEND_WEIGHT_FIELDS])
        h = ctypes.c_void_p()
        check(lib().fsx_append_create(ctypes.byref(self.cfg), ctypes.byref(wst), device, ctypes.byref(h)))
        self.h = h
        del keep

    def close(self):
        if getattr(self, "h", None) and self.h.value:
            lib().fsx_append_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, k_layers, v_layers, offsets, dst_rows, x_new, hidden, stream=None):
        B = int(x_new.shape[0])
        check(lib().fsx_append(self.h, _ptr_array(k_layers), _ptr_array(v_layers), _ptr(offsets), _ptr(dst_rows), B,
                               _ptr(x_new), _ptr(hidden), _stream(stream)))
        return hidden

    def status(self, stream=None) -> int:
        return lib().fsx_append_get_status(self.h, _stream(stream))

    def weight_bytes(self) -> int:
        return int(lib().fsx_append_weight_bytes(self.h))


class Session:
    """An fsx_session: the asynchronous fast-slow schedule of one vehicle over one cache
    (ticks on a snapshot of the committed rows, appends behind them). Marshalling only."""

    def __init__(self, expert: "Expert", append: "Append", k_layers, v_layers, capacity_rows: int,
                 committed_rows: int, concurrent: bool, device: int = 0):
        self._keep = (list(k_layers), list(v_layers))
        h = ctypes.c_void_p()
        check(lib().fsx_session_create(expert.h, append.h, _ptr_array(k_layers), _ptr_array(v_layers),
                                       len(k_layers), append.dims.n_new, capacity_rows, committed_rows,
                                       FSX_SCHED_CONCURRENT if concurrent else FSX_SCHED_SERIAL, device,
                                       ctypes.byref(h)))
        self.h = h

    def close(self):
        if getattr(self, "h", None) and self.h.value:
            lib().fsx_session_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, x_new, hidden):
        check(lib().fsx_session_append(self.h, _ptr(x_new), _ptr(hidden)))

    def tick(self, frames, out) -> int:
        snap = ctypes.c_longlong()
        check(lib().fsx_session_tick(self.h, _ptr(frames), _ptr(out), ctypes.byref(snap)))
        return int(snap.value)

    def committed(self) -> int:
        return int(lib().fsx_session_committed(self.h))

    def reserved(self) -> int:
        return int(lib().fsx_session_reserved(self.h))

    def tick_stream(self) -> int:
        return lib().fsx_session_tick_stream(self.h)

    def append_stream(self) -> int:
        return lib().fsx_session_append_stream(self.h)

    def sync(self):
        check(lib().fsx_session_sync(self.h))
