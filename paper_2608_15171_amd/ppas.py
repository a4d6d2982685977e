"""Thin ctypes binding of libppas.so (C ABI in include/ppas.h).

Argument marshalling only: every step of the computation runs in the library's
HIP kernels. Device buffers are torch tensors (data pointers are passed through),
descriptors and block-table host copies are NumPy int32 arrays. Importing this
module fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libppas.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_15171_amd.build`")

# PyTorch wheels carry their own HIP runtime. Import torch first so that the
# library's libamdhip64.so.7 dependency binds to the runtime torch already
# loaded (same SONAME): device pointers and streams are then shared by one HIP
# runtime. Without torch, the system ROCm runtime is used.
try:
    import torch  # noqa: F401
except ImportError:
    torch = None
_lib = ctypes.CDLL(LIB_PATH)


def _hip_runtimes() -> set:
    paths = set()
    with open("/proc/self/maps") as f:
        for line in f:
            path = line.split()[-1] if len(line.split()) >= 6 else ""
            if os.path.basename(path).startswith("libamdhip64.so"):
                paths.add(os.path.realpath(path))
    return paths


if len(_hip_runtimes()) > 1:
    raise ImportError(f"two HIP runtimes are loaded in this process ({sorted(_hip_runtimes())}); "
                      "import torch before loading libppas.so")

PPAS_OK, PPAS_EINVAL, PPAS_ERANGE, PPAS_ENOSPACE, PPAS_EHIP, PPAS_EUNSUPPORTED = 0, -1, -2, -3, -4, -5


class Shape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("scale", ctypes.c_float)]


class PPASError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


class PlanOpts(ctypes.Structure):
    """Planning choices of one call (0 = automatic): see ppas_plan_opts in include/ppas.h."""
    _fields_ = [("prefill_split", ctypes.c_int32), ("decode_split", ctypes.c_int32),
                ("tile_positions", ctypes.c_int32), ("num_cus", ctypes.c_int32)]


class Events(ctypes.Structure):
    """hipEvent_t handles a call's launches record (None = not recorded): see ppas_events."""
    _fields_ = [("start", ctypes.c_void_p), ("stop", ctypes.c_void_p),
                ("merge_start", ctypes.c_void_p), ("merge_stop", ctypes.c_void_p)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n_items", ctypes.c_int32), ("n_merge", ctypes.c_int32), ("tile_positions", ctypes.c_int32),
                ("n_append", ctypes.c_int32), ("workspace_bytes", ctypes.c_uint64)]


class Rope(ctypes.Structure):
    """Rotary positions in their general form: see ppas_rope in include/ppas.h, and rope() below."""
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("original_len", ctypes.c_int32), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("magnitude", ctypes.c_double)]


class Qkv(ctypes.Structure):
    """A step's new rows where the projection left them: see ppas_qkv."""
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class HeadNorm(ctypes.Structure):
    """The norm of a head before its turn: see ppas_head_norm, and head_norm() below."""
    _fields_ = [("weight", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("eps", ctypes.c_float),
                ("offset", ctypes.c_float), ("center", ctypes.c_int32)]
    tensor = None   # the weights, which head_norm keeps


class Adapters(ctypes.Structure):
    """Low-rank adapters of one projection: see ppas_adapters, and adapters() below."""
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("n_adapters", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("hidden", ctypes.c_int32), ("n_out", ctypes.c_int32)]
    tensors = ()   # the weights, which adapters() keeps


class LogprobOut(ctypes.Structure):
    _fields_ = [("logprob", ctypes.c_void_p), ("rank", ctypes.c_void_p), ("entropy", ctypes.c_void_p),
                ("top_ids", ctypes.c_void_p), ("top_logprobs", ctypes.c_void_p)]


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}

_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_i64, _R = ctypes.c_int64, ctypes.POINTER(Rope)
_P = ctypes.POINTER(Shape)
_O = ctypes.POINTER(PlanOpts)
_E = ctypes.POINTER(Events)
_lib.ppas_status_string.restype = ctypes.c_char_p
_lib.ppas_status_string.argtypes = [ctypes.c_int]
_lib.ppas_validate_step.restype = ctypes.c_int
_lib.ppas_validate_step.argtypes = [_P, _vp, _i32, _vp, _i32]
_lib.ppas_kv_append.restype = ctypes.c_int
_lib.ppas_kv_append.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp]
_lib.ppas_rope_kv_append.restype = ctypes.c_int
_lib.ppas_rope_kv_append.argtypes = [_P, ctypes.c_float, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp]
_lib.ppas_attn_workspace_bytes.restype = _sz
_lib.ppas_attn_workspace_bytes.argtypes = [_P, _vp, _i32]
_lib.ppas_attn_step.restype = ctypes.c_int
_lib.ppas_attn_step.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _sz, _vp]
_lib.ppas_attn_step_noalloc.restype = ctypes.c_int
_lib.ppas_attn_step_noalloc.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp]
_lib.ppas_gateup_proj.restype = ctypes.c_int
_lib.ppas_gateup_proj.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _sz, _E, _vp]
_lib.ppas_gateup_workspace_bytes.restype = _sz
_lib.ppas_gateup_workspace_bytes.argtypes = [_i32, _i32, _i32]
_lib.ppas_gateup_act.restype = ctypes.c_int
_lib.ppas_gateup_act.argtypes = [_vp, _vp, _vp, _i32, _i32, _i32, _vp, _sz, _E, _vp]
_lib.ppas_gateup_act_workspace_bytes.restype = _sz
_lib.ppas_gateup_act_workspace_bytes.argtypes = [_i32, _i32, _i32]
_lib.ppas_gateup_choice.restype = ctypes.c_int
_lib.ppas_gateup_choice.argtypes = [_i32, _i32, _i32, _i32, _i32, _sz, _i32, _vp]
_lib.ppas_gateup_i8_choice.restype = ctypes.c_int
_lib.ppas_gateup_i8_choice.argtypes = [_i32, _i32, _i32, _i32, _i32, _sz, _i32, _vp]
_lib.ppas_stream_read.restype = ctypes.c_int
_lib.ppas_stream_read.argtypes = [_vp, _sz, _vp, _E, _vp]
_lib.ppas_plan_items.restype = _i32
_lib.ppas_plan_items.argtypes = [_P, _vp, _i32, _O, _vp, _i32]
_lib.ppas_plan_shared_items.restype = _i32
_lib.ppas_plan_shared_items.argtypes = [_P, _vp, _i32, _vp, _i32, _O, _vp, _i32]
_lib.ppas_step_plan_create.restype = ctypes.c_int
_lib.ppas_step_plan_create.argtypes = [_P, _vp, _i32, _vp, _i32, _O, ctypes.POINTER(ctypes.c_void_p)]
_lib.ppas_step_plan_info.restype = ctypes.c_int
_lib.ppas_step_plan_info.argtypes = [_vp, ctypes.POINTER(PlanInfo)]
_lib.ppas_step_plan_destroy.restype = None
_lib.ppas_step_plan_destroy.argtypes = [_vp]
_lib.ppas_kv_append_planned.restype = ctypes.c_int
_lib.ppas_kv_append_planned.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _E, _vp]
_lib.ppas_rope_kv_append_planned.restype = ctypes.c_int
_lib.ppas_rope_kv_append_planned.argtypes = [_vp, ctypes.c_float, _vp, _vp, _vp, _vp, _vp, _vp, _E, _vp]
_lib.ppas_attn_step_planned.restype = ctypes.c_int
_lib.ppas_attn_step_planned.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _E, _vp]


_lib.ppas_rope_frequencies.restype = ctypes.c_int
_lib.ppas_rope_frequencies.argtypes = [_R, _i32, _vp]
_lib.ppas_rope_rows.restype = ctypes.c_int
_lib.ppas_rope_rows.argtypes = [_R, _vp, _i64, _vp, _i64, _vp, _i32, _i32, _i32, _i32, _E, _vp]
_lib.ppas_rope_qkv_append.restype = ctypes.c_int
_lib.ppas_rope_qkv_append.argtypes = [_P, _R, ctypes.POINTER(Qkv), _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _vp]
_lib.ppas_rope_qkv_append_planned.restype = ctypes.c_int
_lib.ppas_rope_qkv_append_planned.argtypes = [_vp, _R, ctypes.POINTER(Qkv), _vp, _vp, _vp, _vp, _E, _vp]
_N = ctypes.POINTER(HeadNorm)
_lib.ppas_norm_rope_rows.restype = ctypes.c_int
_lib.ppas_norm_rope_rows.argtypes = [_N, _R, _vp, _i64, _vp, _i64, _vp, _i32, _i32, _i32, _E, _vp]
_lib.ppas_norm_rope_qkv_append.restype = ctypes.c_int
_lib.ppas_norm_rope_qkv_append.argtypes = [_P, _N, _N, _R, ctypes.POINTER(Qkv), _vp, _vp, _vp, _vp, _i32, _vp, _i32,
                                           _vp, _vp]
_lib.ppas_norm_rope_qkv_append_planned.restype = ctypes.c_int
_lib.ppas_norm_rope_qkv_append_planned.argtypes = [_vp, _N, _N, _R, ctypes.POINTER(Qkv), _vp, _vp, _vp, _vp, _E, _vp]
_lib.ppas_step_plan_create_shared.restype = ctypes.c_int
_lib.ppas_step_plan_create_shared.argtypes = [_P, _vp, _i32, _vp, _i32, _vp, _i32, _O, ctypes.POINTER(ctypes.c_void_p)]
_lib.ppas_attn_step_shared.restype = ctypes.c_int
_lib.ppas_attn_step_shared.argtypes = [_P, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _i32, _vp, _i32, _vp, _vp, _sz, _vp]
_lib.ppas_attn_shared_workspace_bytes.restype = _sz
_lib.ppas_attn_shared_workspace_bytes.argtypes = [_P, _vp, _i32, _vp, _i32]
_lib.ppas_quant_i8.restype = ctypes.c_int
_lib.ppas_quant_i8.argtypes = [_vp, _i64, _vp, _vp, _i32, _i32, _E, _vp]
for _f in (_lib.ppas_gateup_proj_i8, _lib.ppas_gateup_act_i8):
    _f.restype = ctypes.c_int
    _f.argtypes = [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _sz, _E, _vp]
for _f in (_lib.ppas_gateup_i8_workspace_bytes, _lib.ppas_gateup_act_i8_workspace_bytes):
    _f.restype = _sz
    _f.argtypes = [_i32, _i32, _i32]
_lib.ppas_adapter_rows_bytes.restype = _sz
_lib.ppas_adapter_rows_bytes.argtypes = [_i32, _i32]
_lib.ppas_adapter_rows.restype = ctypes.c_int
_lib.ppas_adapter_rows.argtypes = [_vp, _i32, _i32, _vp, _sz, _E, _vp]
_lib.ppas_adapter_workspace_bytes.restype = _sz
_lib.ppas_adapter_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32]
for _f in (_lib.ppas_adapter_add, _lib.ppas_adapter_act):
    _f.restype = ctypes.c_int
    _f.argtypes = [ctypes.POINTER(Adapters), _vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _sz, _vp, _sz, _E, _vp]
_lib.ppas_logprobs.restype = ctypes.c_int
_lib.ppas_logprobs.argtypes = [_vp, _i32, _i64, _i32, _i32, ctypes.c_float, _vp, _i32, ctypes.POINTER(LogprobOut), _vp, _sz,
                               _E, _vp]
_lib.ppas_logprobs_workspace_bytes.restype = _sz
_lib.ppas_logprobs_workspace_bytes.argtypes = [_i32, _i32, _i32]


def status_string(status: int) -> str:
    return _lib.ppas_status_string(int(status)).decode()


def make_shape(n_q_heads: int = 16, n_kv_heads: int = 2, num_pages: int = 1, scale: float | None = None,
               head_dim: int = 128, page_size: int = 16) -> Shape:
    if scale is None:
        scale = 1.0 / math.sqrt(head_dim)
    return Shape(n_q_heads, n_kv_heads, head_dim, page_size, num_pages, scale)


def _desc(desc) -> np.ndarray:
    d = np.ascontiguousarray(desc, dtype=np.int32)
    if d.ndim != 2 or d.shape[1] != 3:
        raise ValueError("descriptors must be int32 [S, 3] (query_start, n_query, cached_len)")
    return d


def _host_ptr(a):
    # a third of the time of a.ctypes.data, which makes an object each time
    return None if a is None else a.__array_interface__["data"][0]


def _bt_host(bt_host, bt_dev=None):
    """The host copy of the block table as int32; when the device table is given, the
    two must have the same shape (the library reads the host copy with the device
    table's row stride)."""
    if bt_host is None:
        return None
    bt = np.ascontiguousarray(bt_host, dtype=np.int32)
    if bt.ndim != 2:
        raise ValueError("the host block table must be int32 [n_seqs, stride]")
    if bt_dev is not None and tuple(bt.shape) != tuple(bt_dev.shape):
        raise ValueError(f"host block table {tuple(bt.shape)} and device block table {tuple(bt_dev.shape)} differ")
    return bt


def _dev(t, name):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# bf16 rows: as such, or as their bit patterns
_BF16 = (torch.bfloat16, torch.int16, torch.uint16) if torch is not None else ()


def _is_table(t) -> bool:
    return t.dim() == 2 and t.element_size() == 4 and not t.is_floating_point()


def _rows(d) -> int:
    # plain integers up to where numpy's fixed cost of four small operations is made up:
    # 1 us against 7 at one request, even at about 100
    if len(d) <= 64:
        return sum(n for n in d[:, 1].tolist() if n > 0)
    return int(d[:, 1].astype(np.int64).clip(min=0).sum())


def _need(t, name, nbytes: int, elem: int | None = 2):
    """Refuse a device buffer smaller than the call will touch (or of the wrong
    element size), so a bad argument raises here instead of reaching a kernel."""
    if t is None:
        return
    if elem is not None and t.element_size() != elem:
        raise ValueError(f"{name} must have {elem}-byte elements (bf16 bit patterns), got {t.dtype}")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes; this call needs {nbytes}")


def _check_buffers(shape: Shape, d, q=None, out=None, k_new=None, v_new=None, k_pages=None, v_pages=None,
                   bt_dev=None, rows: int | None = None):
    """`rows`: the step's token rows where the caller has counted them already."""
    if len(d) == 0:
        return                      # an empty step touches no buffer
    T, D = _rows(d) if rows is None else rows, shape.head_dim
    _need(q, "q", T * shape.n_q_heads * D * 2)
    _need(out, "out", T * shape.n_q_heads * D * 2)
    _need(k_new, "k_new", T * shape.n_kv_heads * D * 2)
    _need(v_new, "v_new", T * shape.n_kv_heads * D * 2)
    pool = int(shape.num_pages) * shape.n_kv_heads * shape.page_size * D * 2
    _need(k_pages, "k_pages", pool)
    _need(v_pages, "v_pages", pool)
    if bt_dev is not None:
        if not _is_table(bt_dev):
            raise ValueError("block_table must be an int32 [n_seqs, stride] device tensor")
        if bt_dev.shape[0] < len(d):
            raise ValueError(f"block_table has {bt_dev.shape[0]} rows for {len(d)} requests")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) if torch is not None else None


def _stream(stream):
    if stream is None:
        # the handle itself, without the object around it (1-2 us of a call)
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _here(stream, *tensors):
    """The stream of a call, whose tensors have to live on the current device."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensors of device {t.get_device()}, but the current device is {here}")
    if stream is None and _raw_stream is not None:
        return _raw_stream(here)
    return _stream(stream)


def _check(st: int, what: str):
    if st != PPAS_OK:
        raise PPASError(st, what)


def validate_step(shape: Shape, desc, bt_host=None, bt_stride: int | None = None) -> int:
    d = _desc(desc)
    bt = _bt_host(bt_host)
    stride = bt_stride if bt_stride is not None else (bt.shape[1] if bt is not None else 1)
    return _lib.ppas_validate_step(ctypes.byref(shape), _host_ptr(d), len(d), _host_ptr(bt), stride)


def kv_append(shape: Shape, k_pages, v_pages, k_new, v_new, desc, bt_dev, bt_host=None, stream=None) -> None:
    d = _desc(desc)
    bt = _bt_host(bt_host, bt_dev)
    _check_buffers(shape, d, k_new=k_new, v_new=v_new, k_pages=k_pages, v_pages=v_pages, bt_dev=bt_dev)
    st = _lib.ppas_kv_append(ctypes.byref(shape), _dev(k_pages, "k_pages"), _dev(v_pages, "v_pages"),
                             _dev(k_new, "k_new"), _dev(v_new, "v_new"), _host_ptr(d), len(d),
                             _dev(bt_dev, "block_table"), bt_dev.shape[1], _host_ptr(bt), _stream(stream))
    _check(st, "ppas_kv_append")


def rope_kv_append(shape: Shape, theta: float, q, k_pages, v_pages, k_new, v_new, desc, bt_dev, bt_host=None,
                   stream=None) -> None:
    """Rotate q in place and k_new into the pages at each row's position; copy v_new."""
    d = _desc(desc)
    bt = _bt_host(bt_host, bt_dev)
    _check_buffers(shape, d, q=q, k_new=k_new, v_new=v_new, k_pages=k_pages, v_pages=v_pages, bt_dev=bt_dev)
    st = _lib.ppas_rope_kv_append(ctypes.byref(shape), float(theta), _dev(q, "q"), _dev(k_pages, "k_pages"),
                                  _dev(v_pages, "v_pages"), _dev(k_new, "k_new"), _dev(v_new, "v_new"),
                                  _host_ptr(d), len(d), _dev(bt_dev, "block_table"), bt_dev.shape[1],
                                  _host_ptr(bt), _stream(stream))
    _check(st, "ppas_rope_kv_append")


def rope(layout: str = "half", rotary_dim: int = 128, theta: float = 1e6, scaling: str = "none", factor: float = 1.0,
         original_len: int = 0, low: float = 0.0, high: float = 0.0, magnitude: float = 1.0) -> Rope:
    """Rotary positions: `layout` "half" or "interleaved", the first `rotary_dim` features of a head, frequencies
    scaled for long contexts by "linear", "base", "bands" or "ramp" (ppas_rope in include/ppas.h has the formulas)."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        raise ValueError(f"layout is one of {sorted(ROPE_LAYOUTS)}, scaling one of {sorted(ROPE_SCALINGS)}")
    return Rope(ROPE_LAYOUTS[layout], int(rotary_dim), ROPE_SCALINGS[scaling], int(original_len), float(theta),
                float(factor), float(low), float(high), float(magnitude))


def rope_frequencies(rope: Rope, head_dim: int = 128) -> np.ndarray:
    """Radians per position of every pair (host only)."""
    out = np.zeros(max(int(rope.rotary_dim) // 2, 1), dtype=np.float64)
    _check(_lib.ppas_rope_frequencies(ctypes.byref(rope), int(head_dim), _host_ptr(out)), "ppas_rope_frequencies")
    return out[:int(rope.rotary_dim) // 2]


def _heads(t, name):
    """A device tensor [rows, heads, features] of packed heads (any row stride):
    its data pointer and row stride."""
    if t.dim() != 3 or t.dtype not in _BF16:
        raise ValueError(f"{name} must be [rows, heads, features] of bf16, got {tuple(t.shape)} {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    n, h, d = t.shape
    row, head, one = t.stride()
    if (one != 1 and d > 1) or (head != d and h > 1):
        raise ValueError(f"the heads of {name} must follow each other")
    return t.data_ptr(), row if n > 1 else max(row, h * d)


def _rope_rows_args(x, positions, y):
    """The pointers and strides of rows to turn, their positions and sizes."""
    xp, xs = _heads(x, "x")
    yp, ys = (xp, xs) if y is x else _heads(y, "y")
    shape = x.shape
    if y.shape != shape or positions.shape != shape[:1]:
        raise ValueError(f"shapes x {tuple(x.shape)}, y {tuple(y.shape)}, positions {tuple(positions.shape)} do not match")
    if positions.dtype != torch.int32:
        raise ValueError("positions must be int32")
    return xp, xs, yp, ys, _dev(positions, "positions"), *shape


def rope_rows(rope: Rope, x, positions, y, transposed: bool = False, events: Events | None = None, stream=None) -> None:
    """y[r] = the heads of x[r] turned by positions[r] (x, y [rows, heads, features] bf16 with any row stride,
    positions int32). y may be x. `transposed` turns the other way: the gradient, and without a magnitude the inverse."""
    args = _rope_rows_args(x, positions, y)
    hs = _here(stream, x, y, positions)
    st = _lib.ppas_rope_rows(ctypes.byref(rope), *args, int(bool(transposed)),
                             None if events is None else ctypes.byref(events), hs)
    _check(st, "ppas_rope_rows")


def head_norm(weight=None, eps: float = 1e-6, offset: float = 0.0, center: bool = False) -> HeadNorm:
    """The norm of heads, (x - mu) / sqrt(var + eps) * (offset + weight): `weight` a bf16 device tensor [features] for
    all heads or [heads, features], or None; `center` takes mu as the head's mean (otherwise 0). Keeps the tensor."""
    if weight is not None and not (weight.dtype in _BF16 and 1 <= weight.dim() <= 2 and
                                   (weight.stride(-1) == 1 or weight.shape[-1] == 1)):
        raise ValueError(f"weight must be [features] or [heads, features] of bf16, got {tuple(weight.shape)} {weight.dtype}")
    if weight is not None and not weight.is_cuda:
        raise ValueError("weight must be a device tensor")
    stride = 0
    if weight is not None and weight.dim() == 2:
        stride = weight.stride(0) if weight.shape[0] > 1 else max(weight.stride(0), weight.shape[1])
    n = HeadNorm(None if weight is None else weight.data_ptr(), stride, float(eps), float(offset), int(bool(center)))
    n.tensor = weight
    return n


def _norm(norm: HeadNorm, name, heads: int, dim: int):
    """Refuses a norm whose weights are not of such heads; its weights' tensor (or None)."""
    w = norm.tensor
    if w is not None and w.shape != (dim,) and w.shape != (heads, dim):
        raise ValueError(f"{name}'s weight must be [{dim}] or [{heads}, {dim}], got {tuple(w.shape)}")
    return w


def norm_rope_rows(norm: HeadNorm, rope: Rope, x, positions, y, events: Events | None = None, stream=None) -> None:
    """rope_rows of normalised heads."""
    args = _rope_rows_args(x, positions, y)
    w = _norm(norm, "norm", *args[-2:])
    hs = _here(stream, x, y, positions, w)
    st = _lib.ppas_norm_rope_rows(ctypes.byref(norm), ctypes.byref(rope), *args,
                                  None if events is None else ctypes.byref(events), hs)
    _check(st, "ppas_norm_rope_rows")


def _step_rows(t, name, rows: int, heads: int, dim: int):
    """_heads of at least `rows` rows of `heads` heads of `dim` features."""
    p = _heads(t, name)
    n, h, d = t.shape
    if n < rows or h != heads or d != dim:
        raise ValueError(f"{name} must be [{rows} rows or more, {heads}, {dim}], got {tuple(t.shape)}")
    return p


def _qkv(q, k, v, rows: int, hq: int, hkv: int, dim: int) -> Qkv:
    """The step's rows as ppas_qkv."""
    qp, qs = _step_rows(q, "q_new", rows, hq, dim)
    kp, ks = _step_rows(k, "k_new", rows, hkv, dim)
    vp, vs = _step_rows(v, "v_new", rows, hkv, dim)
    return Qkv(qp, kp, vp, qs, ks, vs)


def _buffer(t, name, nbytes: int):
    """_need and _dev in one: the pointer of a contiguous device buffer of bf16."""
    if t.dtype not in _BF16:
        raise ValueError(f"{name} must be bf16, got {t.dtype}")
    if t.numel() * 2 < nbytes or not t.is_cuda or not t.is_contiguous():
        _need(t, name, nbytes)
        _dev(t, name)
    return t.data_ptr()


def _qkv_append(fn, what, shape, norms, rope, q, k_pages, v_pages, q_new, k_new, v_new, desc, bt_dev, bt_host, stream):
    d = _desc(desc)
    bt = _bt_host(bt_host, bt_dev)
    rows = _rows(d)
    _check_buffers(shape, d, bt_dev=bt_dev)
    x = _qkv(q_new, k_new, v_new, rows, shape.n_q_heads, shape.n_kv_heads, shape.head_dim)
    pool = int(shape.num_pages) * shape.n_kv_heads * shape.page_size * shape.head_dim * 2 if len(d) else 0
    ptrs = (_buffer(q, "q", rows * shape.n_q_heads * shape.head_dim * 2), _buffer(k_pages, "k_pages", pool),
            _buffer(v_pages, "v_pages", pool), _dev(bt_dev, "block_table"))
    weights = [_norm(n, name, h, shape.head_dim)
               for n, name, h in zip(norms, ("q_norm", "k_norm"), (shape.n_q_heads, shape.n_kv_heads))]
    hs = _here(stream, q, k_pages, v_pages, q_new, k_new, v_new, bt_dev, *weights)
    st = fn(ctypes.byref(shape), *map(ctypes.byref, norms), ctypes.byref(rope), ctypes.byref(x), *ptrs[:3], _host_ptr(d),
            len(d), ptrs[3], bt_dev.shape[1], _host_ptr(bt), hs)
    _check(st, what)


def rope_qkv_append(shape: Shape, rope: Rope, q, k_pages, v_pages, q_new, k_new, v_new, desc, bt_dev, bt_host=None,
                    stream=None) -> None:
    """Rotate the rows q_new into q and k_new into the pages at their positions, and copy v_new into the pages. The
    rows are [T, heads, 128] at any row stride, as a fused QKV projection leaves them."""
    _qkv_append(_lib.ppas_rope_qkv_append, "ppas_rope_qkv_append", shape, (), rope, q, k_pages, v_pages, q_new, k_new,
                v_new, desc, bt_dev, bt_host, stream)


def norm_rope_qkv_append(shape: Shape, q_norm: HeadNorm, k_norm: HeadNorm, rope: Rope, q, k_pages, v_pages, q_new, k_new,
                         v_new, desc, bt_dev, bt_host=None, stream=None) -> None:
    """rope_qkv_append of normalised query and key heads."""
    _qkv_append(_lib.ppas_norm_rope_qkv_append, "ppas_norm_rope_qkv_append", shape, (q_norm, k_norm), rope, q, k_pages,
                v_pages, q_new, k_new, v_new, desc, bt_dev, bt_host, stream)


def _prefixes(prefixes):
    """Shared prefixes as int32 [P, 3] rows of (first request, requests, positions), or None."""
    if prefixes is None or len(prefixes) == 0:
        return None
    given = np.asarray(prefixes)
    p = np.ascontiguousarray(given, dtype=np.int32)
    if p.ndim != 2 or p.shape[1] != 3 or (given.dtype != np.int32 and not np.array_equal(p, given)):
        raise ValueError("prefixes must be int32 [P, 3] (first_seq, n_seqs, len)")
    return p


def attn_shared_workspace_bytes(shape: Shape, desc, prefixes) -> int:
    d, p = _desc(desc), _prefixes(prefixes)
    return int(_lib.ppas_attn_shared_workspace_bytes(ctypes.byref(shape), _host_ptr(d), len(d), _host_ptr(p),
                                                     0 if p is None else len(p)))


def attn_step_shared(shape: Shape, out, q, k_pages, v_pages, desc, prefixes, bt_dev, workspace, bt_host=None,
                     stream=None) -> None:
    """attn_step for a step whose requests share prefixes: rows (first request, requests, shared positions)."""
    d, p = _desc(desc), _prefixes(prefixes)
    bt = _bt_host(bt_host, bt_dev)
    if len(d) == 0 or not _is_table(bt_dev) or bt_dev.shape[0] < len(d):
        _check_buffers(shape, d, bt_dev=bt_dev)
        rows, pool = 0, 0
    else:
        rows = _rows(d) * shape.n_q_heads * shape.head_dim * 2
        pool = int(shape.num_pages) * shape.n_kv_heads * shape.page_size * shape.head_dim * 2
    ptrs = (_buffer(out, "out", rows), _buffer(q, "q", rows), _buffer(k_pages, "k_pages", pool),
            _buffer(v_pages, "v_pages", pool), _dev(bt_dev, "block_table"), _dev(workspace, "workspace"))
    hs = _here(stream, out, q, k_pages, v_pages, bt_dev, workspace)
    st = _lib.ppas_attn_step_shared(ctypes.byref(shape), *ptrs[:4], _host_ptr(d), len(d), _host_ptr(p),
                                    0 if p is None else len(p), ptrs[4], bt_dev.shape[1], _host_ptr(bt), ptrs[5],
                                    workspace.numel() * workspace.element_size(), hs)
    _check(st, "ppas_attn_step_shared")


def attn_workspace_bytes(shape: Shape, desc) -> int:
    d = _desc(desc)
    return int(_lib.ppas_attn_workspace_bytes(ctypes.byref(shape), _host_ptr(d), len(d)))


def attn_step(shape: Shape, out, q, k_pages, v_pages, desc, bt_dev, workspace, bt_host=None, stream=None) -> None:
    d = _desc(desc)
    bt = _bt_host(bt_host, bt_dev)
    _check_buffers(shape, d, q=q, out=out, k_pages=k_pages, v_pages=v_pages, bt_dev=bt_dev)
    st = _lib.ppas_attn_step(ctypes.byref(shape), _dev(out, "out"), _dev(q, "q"), _dev(k_pages, "k_pages"),
                             _dev(v_pages, "v_pages"), _host_ptr(d), len(d), _dev(bt_dev, "block_table"),
                             bt_dev.shape[1], _host_ptr(bt), _dev(workspace, "workspace"),
                             workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "ppas_attn_step")


def attn_step_noalloc(shape: Shape, out, q, k_pages, v_pages, desc, bt_dev, bt_host=None, stream=None) -> None:
    """ppas_attn_step without a workspace: the library's fixed device array holds the work list
    and the split partials (PPAS_ENOSPACE when the step does not fit it)."""
    d = _desc(desc)
    bt = _bt_host(bt_host, bt_dev)
    _check_buffers(shape, d, q=q, out=out, k_pages=k_pages, v_pages=v_pages, bt_dev=bt_dev)
    st = _lib.ppas_attn_step_noalloc(ctypes.byref(shape), _dev(out, "out"), _dev(q, "q"), _dev(k_pages, "k_pages"),
                                     _dev(v_pages, "v_pages"), _host_ptr(d), len(d), _dev(bt_dev, "block_table"),
                                     bt_dev.shape[1], _host_ptr(bt), _stream(stream))
    _check(st, "ppas_attn_step_noalloc")


def gateup_workspace_bytes(n_tokens: int, hidden: int, n_out: int) -> int:
    return int(_lib.ppas_gateup_workspace_bytes(int(n_tokens), int(hidden), int(n_out)))


def gateup_proj(x, w, y, workspace=None, events: Events | None = None, stream=None) -> None:
    """y = x w^T: the fused gate-up projection (x [T, H], w [N, H], y [T, N], bf16 device tensors).
    workspace: a device buffer for split reductions (see gateup_workspace_bytes), or None."""
    for t, name in ((x, "x"), (w, "w"), (y, "y")):
        if t.dim() != 2 or t.element_size() != 2:
            raise ValueError(f"{name} must be a 2-D bf16 tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    T, H = x.shape
    N = w.shape[0]
    if w.shape[1] != H or tuple(y.shape) != (T, N):
        raise ValueError(f"shapes x {tuple(x.shape)}, w {tuple(w.shape)}, y {tuple(y.shape)} do not match")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.ppas_gateup_proj(_dev(x, "x"), _dev(w, "w"), _dev(y, "y"), T, H, N, _dev(workspace, "workspace"),
                               ws_bytes, None if events is None else ctypes.byref(events), _stream(stream))
    _check(st, "ppas_gateup_proj")


def gateup_choice(n_tokens: int, hidden: int, n_out: int, activation: bool = False, aligned: bool = True,
                  workspace_bytes: int | None = None, num_cus: int = 0) -> dict:
    """The kernel a projection call takes (host only, for tests); workspace_bytes: None = as many as it can use."""
    out = np.zeros(8, dtype=np.int32)
    nbytes = (1 << 62) if workspace_bytes is None else int(workspace_bytes)
    _check(_lib.ppas_gateup_choice(int(n_tokens), int(hidden), int(n_out), int(activation), int(aligned), nbytes,
                                   int(num_cus), _host_ptr(out)), "ppas_gateup_choice")
    names = ("kernel", "rows", "main_tiles", "small_tiles", "weight_tiles", "weight_rows", "splits",
             "block")
    c = dict(zip(names, out.tolist()))
    c["kernel"] = ("tiles", "rows", "general")[c["kernel"]]
    return c


def gateup_act_workspace_bytes(n_tokens: int, hidden: int, n_inter: int) -> int:
    return int(_lib.ppas_gateup_act_workspace_bytes(int(n_tokens), int(hidden), int(n_inter)))


def gateup_act(x, w, y, workspace=None, events: Events | None = None, stream=None) -> None:
    """y = silu(x w_gate^T) * (x w_up^T): the gate-up projection with the gated activation
    (x [T, H], w [2I, H] with the gate rows over the up rows, y [T, I], bf16 device tensors).
    workspace: a device buffer for split reductions (see gateup_act_workspace_bytes), or None."""
    for t, name in ((x, "x"), (w, "w"), (y, "y")):
        if t.dim() != 2 or t.element_size() != 2:
            raise ValueError(f"{name} must be a 2-D bf16 tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    T, H = x.shape
    N = w.shape[0]
    if N % 2 or w.shape[1] != H or tuple(y.shape) != (T, N // 2):
        raise ValueError(f"shapes x {tuple(x.shape)}, w {tuple(w.shape)}, y {tuple(y.shape)} do not match")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib.ppas_gateup_act(_dev(x, "x"), _dev(w, "w"), _dev(y, "y"), T, H, N // 2, _dev(workspace, "workspace"),
                              ws_bytes, None if events is None else ctypes.byref(events), _stream(stream))
    _check(st, "ppas_gateup_act")


def quant_i8(x, xq, scale, events: Events | None = None, stream=None) -> None:
    """The rows of x [R, H] (bf16, any row stride) as 8-bit integers xq [R, H] (int8) and a scale each (fp32 [R]):
    token rows of activations, or output channels of weights."""
    if x.dim() != 2 or x.dtype not in _BF16 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"x must be a 2-D bf16 tensor of packed rows, got {tuple(x.shape)} {x.dtype}")
    R, H = x.shape
    if tuple(xq.shape) != (R, H) or xq.dtype != torch.int8 or tuple(scale.shape) != (R,) or scale.dtype != torch.float32:
        raise ValueError(f"xq must be int8 {(R, H)} and scale fp32 {(R,)}, got {tuple(xq.shape)} {xq.dtype} and "
                         f"{tuple(scale.shape)} {scale.dtype}")
    if not x.is_cuda:
        raise ValueError("x must be a device tensor")
    qp, sp = _dev(xq, "xq"), _dev(scale, "scale")
    hs = _here(stream, x, xq, scale)
    st = _lib.ppas_quant_i8(x.data_ptr(), x.stride(0) if R > 1 else max(x.stride(0), H), qp, sp, R, H,
                            None if events is None else ctypes.byref(events), hs)
    _check(st, "ppas_quant_i8")


def gateup_i8_workspace_bytes(n_tokens: int, hidden: int, n_out: int) -> int:
    return int(_lib.ppas_gateup_i8_workspace_bytes(int(n_tokens), int(hidden), int(n_out)))


def gateup_act_i8_workspace_bytes(n_tokens: int, hidden: int, n_inter: int) -> int:
    return int(_lib.ppas_gateup_act_i8_workspace_bytes(int(n_tokens), int(hidden), int(n_inter)))


def gateup_i8_choice(n_tokens: int, hidden: int, n_out: int, activation: bool = False, aligned: bool = True,
                     workspace_bytes: int | None = None, num_cus: int = 0) -> list:
    """The launches of an 8-bit product (host only, for tests), one or two; n_out: its weight rows."""
    out = np.zeros(16, dtype=np.int32)
    nbytes = (1 << 62) if workspace_bytes is None else int(workspace_bytes)
    _check(_lib.ppas_gateup_i8_choice(int(n_tokens), int(hidden), int(n_out), int(activation), int(aligned), nbytes,
                                      int(num_cus), _host_ptr(out)), "ppas_gateup_i8_choice")
    names = ("tokens", "kernel", "rows", "main_tiles", "small_tiles", "weight_tiles", "weight_rows", "splits")
    launches = [dict(zip(names, out[i:i + 8].tolist())) for i in (0, 8) if out[i] > 0]
    for c in launches:
        c["kernel"] = ("tiles", "rows", "general", "mid")[c["kernel"]]
    return launches


def _gateup_i8(fn, what, x, x_scale, w, w_scale, y, per, workspace, events, stream):
    if not (x.dim() == w.dim() == y.dim() == 2 and x.dtype == w.dtype == torch.int8 and y.dtype in _BF16):
        raise ValueError(f"x and w must be 2-D int8 tensors and y a 2-D bf16 tensor, got {x.dtype}, {w.dtype}, {y.dtype}")
    T, H = x.shape
    N = w.shape[0]
    if N % per or w.shape[1] != H or tuple(y.shape) != (T, N // per):
        raise ValueError(f"shapes x {tuple(x.shape)}, w {tuple(w.shape)}, y {tuple(y.shape)} do not match")
    if not (x_scale.numel() == T and w_scale.numel() == N and x_scale.dtype == w_scale.dtype == torch.float32):
        raise ValueError(f"x_scale must hold {T} fp32 values and w_scale {N}")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    xp, sp, wp, vp, yp = (_dev(x, "x"), _dev(x_scale, "x_scale"), _dev(w, "w"), _dev(w_scale, "w_scale"), _dev(y, "y"))
    ws = _dev(workspace, "workspace")
    hs = _here(stream, x, x_scale, w, w_scale, y, workspace)
    st = fn(xp, sp, wp, vp, yp, T, H, N // per, ws, ws_bytes, None if events is None else ctypes.byref(events), hs)
    _check(st, what)


def gateup_proj_i8(x, x_scale, w, w_scale, y, workspace=None, events: Events | None = None, stream=None) -> None:
    """y = (x x_scale) (w w_scale)^T for 8-bit rows x [T, H] and w [N, H] with fp32 scales per row; y [T, N] bf16.
    workspace: a device buffer for split reductions (see gateup_i8_workspace_bytes), or None."""
    _gateup_i8(_lib.ppas_gateup_proj_i8, "ppas_gateup_proj_i8", x, x_scale, w, w_scale, y, 1, workspace, events, stream)


def gateup_act_i8(x, x_scale, w, w_scale, y, workspace=None, events: Events | None = None, stream=None) -> None:
    """The gated activation of such products, as gateup_act (w [2I, H], y [T, I]).
    workspace: see gateup_act_i8_workspace_bytes, or None."""
    _gateup_i8(_lib.ppas_gateup_act_i8, "ppas_gateup_act_i8", x, x_scale, w, w_scale, y, 2, workspace, events, stream)


class AdapterRows:
    """A step's rows in the order of their adapters (ppas_adapter_rows), in device memory of its own: sorted once per step,
    used by every adapter_add and adapter_act of the step."""

    def __init__(self, n_tokens: int, n_adapters: int, device="cuda"):
        self.n_tokens, self.n_adapters, self.sorted = int(n_tokens), int(n_adapters), False
        size = int(_lib.ppas_adapter_rows_bytes(self.n_tokens, self.n_adapters))
        if size == 0 and self.n_tokens != 0:
            raise ValueError(f"no rows of {self.n_tokens} tokens and {self.n_adapters} adapters")
        self.buf = torch.empty(max(size, 16), dtype=torch.uint8, device=device)
        self._at = self.buf.data_ptr(), self.buf.numel()   # as the calls take it

    def sort(self, row_adapter, events: Events | None = None, stream=None) -> None:
        """row_adapter: int32 [n_tokens], the rows' adapters (-1: none)."""
        if row_adapter.dtype != torch.int32 or row_adapter.shape != (self.n_tokens,):
            raise ValueError(f"row_adapter must be int32 [{self.n_tokens}], got {row_adapter.dtype} {tuple(row_adapter.shape)}")
        p = _dev(row_adapter, "row_adapter")
        hs = _here(stream, row_adapter, self.buf)
        st = _lib.ppas_adapter_rows(p, self.n_tokens, self.n_adapters, *self._at,
                                    None if events is None else ctypes.byref(events), hs)
        _check(st, "ppas_adapter_rows")
        self.sorted = True


def adapters(a, b, scale=None) -> Adapters:
    """Low-rank adapters of one projection: a [n, rank, hidden] and b [n, out, rank] bf16, scale fp32 [n] or None (1).
    Keeps the tensors."""
    if not (a.dim() == b.dim() == 3 and a.dtype in _BF16 and b.dtype in _BF16 and a.shape[0] == b.shape[0] and
            a.shape[1] == b.shape[2]):
        raise ValueError(f"a must be [n, rank, hidden] and b [n, out, rank] of bf16, got {tuple(a.shape)} {a.dtype} and "
                         f"{tuple(b.shape)} {b.dtype}")
    n, r, h = a.shape
    if scale is not None and (scale.dtype != torch.float32 or tuple(scale.shape) != (n,)):
        raise ValueError(f"scale must be fp32 [{n}], got {scale.dtype} {tuple(scale.shape)}")
    s = Adapters(_dev(a, "a"), _dev(b, "b"), _dev(scale, "scale"), n, r, h, b.shape[1])
    s.tensors = (a, b) if scale is None else (a, b, scale)
    return s


def adapter_workspace_bytes(n_tokens: int, hidden: int, rank: int, n_adapters: int) -> int:
    return int(_lib.ppas_adapter_workspace_bytes(int(n_tokens), int(hidden), int(rank), int(n_adapters)))


def _packed_rows(t, name, rows: int, cols: int):
    """The pointer and row stride of a device tensor [rows, cols] of bf16 with packed rows at any stride."""
    if t.shape != (rows, cols) or t.dtype not in _BF16:
        raise ValueError(f"{name} must be bf16 [{rows}, {cols}], got {tuple(t.shape)} {t.dtype}")
    row, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"the rows of {name} must be packed")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return t.data_ptr(), row if rows > 1 else max(row, cols)


def _adapt(fn, what, adapters, x, y, out, rows, per, workspace, events, stream):
    if x.dim() != 2:
        raise ValueError(f"x must be 2-D, got {tuple(x.shape)}")
    T, N = x.shape[0], adapters.n_out
    if rows.n_tokens != T or rows.n_adapters != adapters.n_adapters:
        raise ValueError(f"rows are of {rows.n_tokens} tokens and {rows.n_adapters} adapters, the call of {T} and "
                         f"{adapters.n_adapters}")
    if not rows.sorted:
        raise ValueError("rows have not been sorted")
    if N % per:
        raise ValueError(f"{N} outputs are not a gate and an up half")
    ptrs = (*_packed_rows(x, "x", T, adapters.hidden), *_packed_rows(y, "y", T, N), *_packed_rows(out, "out", T, N // per))
    ws = _dev(workspace, "workspace")
    hs = _here(stream, x, y, out, workspace, rows.buf, *adapters.tensors)
    st = fn(ctypes.byref(adapters), *ptrs, T, *rows._at, ws, workspace.nbytes,
            None if events is None else ctypes.byref(events), hs)
    _check(st, what)


def adapter_add(adapters: Adapters, x, y, out, rows: AdapterRows, workspace, events: Events | None = None, stream=None) -> None:
    """out = y with the adapters' share of its rows: x [T, hidden] the projection's input, y and out [T, n_out] (bf16 rows at
    any stride; out may be y). workspace: a device buffer of adapter_workspace_bytes; one made for a larger step serves a
    smaller one too."""
    _adapt(_lib.ppas_adapter_add, "ppas_adapter_add", adapters, x, y, out, rows, 1, workspace, events, stream)


def adapter_act(adapters: Adapters, x, y, out, rows: AdapterRows, workspace, events: Events | None = None, stream=None) -> None:
    """out [T, n_out / 2] = silu(g) * u of the halves g and u of y with the adapters' share; otherwise as adapter_add."""
    _adapt(_lib.ppas_adapter_act, "ppas_adapter_act", adapters, x, y, out, rows, 2, workspace, events, stream)


def logprobs_workspace_bytes(n_rows: int, vocab: int, top_k: int = 0) -> int:
    return int(_lib.ppas_logprobs_workspace_bytes(int(n_rows), int(vocab), int(top_k)))


def _result(t, name, dtype, *shape):
    """The pointer of an optional result of that type and shape (its device is _here's to check)."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def logprobs(logits, tokens=None, logprob=None, rank=None, entropy=None, top_ids=None, top_logprobs=None, scale: float = 1.0,
             workspace=None, events: Events | None = None, stream=None) -> None:
    """Log probabilities from logits [R, V] (bf16 or fp32, any row stride), times `scale`: into logprob (fp32 [R]) and rank
    (int32 [R]) those of tokens (int32 [R]), into entropy (fp32 [R]) the rows', into top_ids (int32 [R, k]) and top_logprobs
    (fp32 [R, k]) the top k tokens. Results that are None are left out. workspace: see logprobs_workspace_bytes, or None."""
    f32, i32 = torch.float32, torch.int32
    wide = logits.dtype == f32
    if logits.dim() != 2 or not (wide or logits.dtype in _BF16):
        raise ValueError(f"logits must be 2-D bf16 or fp32 rows, got {tuple(logits.shape)} {logits.dtype}")
    R, V = logits.shape
    row, one = logits.stride()
    if one != 1 and V > 1:
        raise ValueError("the rows of logits must be packed")
    top = top_logprobs if top_ids is None else top_ids
    k = top.shape[-1] if top is not None and top.dim() > 0 else 0
    tp = _result(tokens, "tokens", i32, R)
    out = LogprobOut(_result(logprob, "logprob", f32, R), _result(rank, "rank", i32, R), _result(entropy, "entropy", f32, R),
                     _result(top_ids, "top_ids", i32, R, k), _result(top_logprobs, "top_logprobs", f32, R, k))
    if not logits.is_cuda:
        raise ValueError("logits must be a device tensor")
    ws = _dev(workspace, "workspace")
    hs = _here(stream, logits, tokens, logprob, rank, entropy, top_ids, top_logprobs, workspace)
    st = _lib.ppas_logprobs(logits.data_ptr(), int(wide), row if R > 1 else max(row, V), R, V, float(scale), tp, k,
                            ctypes.byref(out), ws,
                            0 if workspace is None else workspace.nbytes, None if events is None else ctypes.byref(events), hs)
    _check(st, "ppas_logprobs")


def stream_read(buf, sink, events: Events | None = None, stream=None) -> None:
    """A plain streaming read of the whole of `buf` (a contiguous device tensor, a multiple of
    16 bytes): the XOR of its 16-byte words, as four 32-bit lanes, is XORed into `sink` (a
    device tensor of 16 bytes). The measured HBM read ceiling of the device."""
    nbytes = buf.numel() * buf.element_size()
    if sink.numel() * sink.element_size() != 16:
        raise ValueError("sink must hold 16 bytes")
    st = _lib.ppas_stream_read(_dev(buf, "buf"), nbytes, _dev(sink, "sink"),
                               None if events is None else ctypes.byref(events), _stream(stream))
    _check(st, "ppas_stream_read")


def plan_opts(prefill_split: int = 0, decode_split: int = 0, tile_positions: int = 0, num_cus: int = 0) -> PlanOpts:
    return PlanOpts(int(prefill_split), int(decode_split), int(tile_positions), int(num_cus))


def events(start=None, stop=None, merge_start=None, merge_stop=None) -> Events:
    return Events(start, stop, merge_start, merge_stop)


def _opts_ptr(opts):
    return None if opts is None else ctypes.byref(opts)


def plan_items(shape: Shape, desc, num_cus: int = 256, opts: PlanOpts | None = None, prefixes=None) -> np.ndarray:
    """The planned work list as int32 [n, 8]: kind, seq, kv_head, row0, pos0, npos, key_lo, key_hi (with prefixes: see
    ppas_plan_shared_items)."""
    d, p = _desc(desc), _prefixes(prefixes)
    o = PlanOpts() if opts is None else PlanOpts(opts.prefill_split, opts.decode_split, opts.tile_positions,
                                                 opts.num_cus)
    if o.num_cus == 0:
        o.num_cus = int(num_cus)
    args = ctypes.byref(shape), _host_ptr(d), len(d), _host_ptr(p), 0 if p is None else len(p), ctypes.byref(o)
    n = _lib.ppas_plan_shared_items(*args, None, 0)
    if n < 0:
        raise PPASError(n, "ppas_plan_shared_items")
    out = np.zeros((max(n, 1), 8), dtype=np.int32)
    _lib.ppas_plan_shared_items(*args, out.ctypes.data, n)
    return out[:n]


class StepPlan:
    """A step's validated descriptors, attention work list and page-write list, made once
    (ppas_step_plan_create) and used by any number of planned calls, e.g. one per layer."""

    def __init__(self, shape: Shape, desc, bt_host=None, bt_stride: int | None = None, opts: PlanOpts | None = None,
                 prefixes=None):
        """prefixes: rows (first request, requests, shared positions) of requests that share their first pages."""
        self.shape = Shape(shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.page_size, shape.num_pages,
                           shape.scale)
        self.desc = _desc(desc)
        self._n_rows = _rows(self.desc)   # counted once: a planned call is made for every layer
        s = self.shape
        self._heads = s.n_q_heads, s.n_kv_heads, s.head_dim
        self._q_bytes = self._n_rows * s.n_q_heads * s.head_dim * 2
        self._pool_bytes = int(s.num_pages) * s.n_kv_heads * s.page_size * s.head_dim * 2
        bt = _bt_host(bt_host)
        self.bt_stride = int(bt_stride if bt_stride is not None else (bt.shape[1] if bt is not None else 1))
        if bt is not None and bt.shape[1] != self.bt_stride:
            raise ValueError("bt_stride differs from the host block table's row length")
        h = ctypes.c_void_p()
        p = _prefixes(prefixes)
        if p is None:
            st = _lib.ppas_step_plan_create(ctypes.byref(self.shape), _host_ptr(self.desc), len(self.desc),
                                            _host_ptr(bt), self.bt_stride, _opts_ptr(opts), ctypes.byref(h))
            _check(st, "ppas_step_plan_create")
        else:
            st = _lib.ppas_step_plan_create_shared(ctypes.byref(self.shape), _host_ptr(self.desc), len(self.desc),
                                                   _host_ptr(p), len(p), _host_ptr(bt), self.bt_stride,
                                                   _opts_ptr(opts), ctypes.byref(h))
            _check(st, "ppas_step_plan_create_shared")
        self._h = h.value
        self._shared = p is not None
        self.info = PlanInfo()
        _check(_lib.ppas_step_plan_info(self._h, ctypes.byref(self.info)), "ppas_step_plan_info")

    @property
    def workspace_bytes(self) -> int:
        return int(self.info.workspace_bytes)

    def _bt(self, bt_dev):
        if bt_dev is None:
            raise ValueError("block_table is required")
        if bt_dev.dim() != 2 or bt_dev.shape[1] != self.bt_stride:
            raise ValueError(f"block_table must have rows of {self.bt_stride} entries, got {tuple(bt_dev.shape)}")
        return bt_dev

    def kv_append(self, k_pages, v_pages, k_new, v_new, bt_dev, events: Events | None = None, stream=None) -> None:
        _check_buffers(self.shape, self.desc, k_new=k_new, v_new=v_new, k_pages=k_pages, v_pages=v_pages,
                       bt_dev=self._bt(bt_dev), rows=self._n_rows)
        st = _lib.ppas_kv_append_planned(self._h, _dev(k_pages, "k_pages"), _dev(v_pages, "v_pages"),
                                         _dev(k_new, "k_new"), _dev(v_new, "v_new"), _dev(bt_dev, "block_table"),
                                         None if events is None else ctypes.byref(events), _stream(stream))
        _check(st, "ppas_kv_append_planned")

    def rope_kv_append(self, theta: float, q, k_pages, v_pages, k_new, v_new, bt_dev, events: Events | None = None,
                       stream=None) -> None:
        _check_buffers(self.shape, self.desc, q=q, k_new=k_new, v_new=v_new, k_pages=k_pages, v_pages=v_pages,
                       bt_dev=self._bt(bt_dev), rows=self._n_rows)
        st = _lib.ppas_rope_kv_append_planned(self._h, float(theta), _dev(q, "q"), _dev(k_pages, "k_pages"),
                                              _dev(v_pages, "v_pages"), _dev(k_new, "k_new"), _dev(v_new, "v_new"),
                                              _dev(bt_dev, "block_table"),
                                              None if events is None else ctypes.byref(events), _stream(stream))
        _check(st, "ppas_rope_kv_append_planned")

    def _qkv_append(self, fn, what, norms, rope, q, k_pages, v_pages, q_new, k_new, v_new, bt_dev, events, stream) -> None:
        bt = self._bt(bt_dev)
        if (bt.dtype != torch.int32 and not _is_table(bt)) or bt.shape[0] < len(self.desc):
            _check_buffers(self.shape, self.desc, bt_dev=bt)
        hq, hkv, dim = self._heads
        x = _qkv(q_new, k_new, v_new, self._n_rows, hq, hkv, dim)
        ptrs = (_buffer(q, "q", self._q_bytes), _buffer(k_pages, "k_pages", self._pool_bytes),
                _buffer(v_pages, "v_pages", self._pool_bytes), _dev(bt, "block_table"))
        weights, refs = (), ()
        if norms:
            qn, kn = norms
            weights = _norm(qn, "q_norm", hq, dim), _norm(kn, "k_norm", hkv, dim)
            refs = ctypes.byref(qn), ctypes.byref(kn)
        hs = _here(stream, q, k_pages, v_pages, q_new, k_new, v_new, bt, *weights)
        st = fn(self._h, *refs, ctypes.byref(rope), ctypes.byref(x), *ptrs,
                None if events is None else ctypes.byref(events), hs)
        _check(st, what)

    def rope_qkv_append(self, rope: Rope, q, k_pages, v_pages, q_new, k_new, v_new, bt_dev,
                        events: Events | None = None, stream=None) -> None:
        self._qkv_append(_lib.ppas_rope_qkv_append_planned, "ppas_rope_qkv_append_planned", (), rope, q, k_pages,
                         v_pages, q_new, k_new, v_new, bt_dev, events, stream)

    def norm_rope_qkv_append(self, q_norm: HeadNorm, k_norm: HeadNorm, rope: Rope, q, k_pages, v_pages, q_new, k_new,
                             v_new, bt_dev, events: Events | None = None, stream=None) -> None:
        self._qkv_append(_lib.ppas_norm_rope_qkv_append_planned, "ppas_norm_rope_qkv_append_planned", (q_norm, k_norm),
                         rope, q, k_pages, v_pages, q_new, k_new, v_new, bt_dev, events, stream)

    def attn_step(self, out, q, k_pages, v_pages, bt_dev, workspace, events: Events | None = None,
                  stream=None) -> None:
        _check_buffers(self.shape, self.desc, q=q, out=out, k_pages=k_pages, v_pages=v_pages,
                       bt_dev=self._bt(bt_dev), rows=self._n_rows)
        hs = _here(stream, out, q, k_pages, v_pages, bt_dev, workspace) if self._shared else _stream(stream)
        st = _lib.ppas_attn_step_planned(self._h, _dev(out, "out"), _dev(q, "q"), _dev(k_pages, "k_pages"),
                                         _dev(v_pages, "v_pages"), _dev(bt_dev, "block_table"),
                                         _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                         None if events is None else ctypes.byref(events), hs)
        _check(st, "ppas_attn_step_planned")

    def close(self) -> None:
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.ppas_step_plan_destroy(h)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        self.close()
