"""ctypes binding of ``libgws.so``: argument marshalling only.

Function names and argument order mirror ``include/gws.h``.  torch is used for
device memory and streams; every step of the method runs in the library's HIP
kernels.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("GWS_LIBRARY") or os.path.join(_HERE, "libgws.so")

FMT_BF16, FMT_FP8_E4M3, FMT_FP6_E3M2 = 0, 1, 2
LINEAR_AUTO, LINEAR_IN_OPERAND, LINEAR_TWO_KERNELS = 0, 2, 3
BASIS_BITS, BASIS_UNIFORM_BF16, BASIS_BOX_MULLER = 0, 1, 2
ACT_SILU, ACT_GELU_TANH, ACT_NONE = 0, 1, 2
NORM_LAYER, NORM_RMS = 0, 1
GATED_FWD, GATED_BWD, GATED_BWD_X = 0, 1, 2                                          # of gws_gated_form: the call,
GATED_ANY, GATED_STREAM, GATED_MIDDLE, GATED_LARGE, GATED_SHARED = 1, 2, 3, 4, 5     # and its kernel

# include/gws.h (the method) and include/gws_bench.h (measurement aids)
EXPORTS = ("gws_sample_fwd", "gws_sample_bwd", "gws_sample_fwd_bi", "gws_sample_bwd_bi", "gws_sample_fwd_mx", "gws_linear_fwd", "gws_linear_fwd_mode",
           "gws_linear_fwd_ws", "gws_linear_fwd_workspace_bytes", "gws_linear_fwd_static", "gws_linear_bwd_w", "gws_linear_bwd_w_ws", "gws_linear_bwd_w_workspace_bytes", "gws_gemm_bf16", "gws_gemm_bf16_sample_next", "gws_gemm_bf16_sample_next_n", "gws_noise_packed",
           "gws_sample_fwd_basis", "gws_sample_bwd_basis", "gws_noise_basis",
           "gws_act8_encode", "gws_act8_decode", "gws_gated_fwd", "gws_gated_bwd", "gws_gated_bwd_h", "gws_gated_bwd_x",
           "gws_linear_bwd_w_act8", "gws_linear_bwd_w_act8_workspace_bytes",
           "gws_norm_fwd", "gws_norm_bwd", "gws_norm_bwd_workspace_bytes", "gws_dense_fwd", "gws_dense_bwd", "gws_dense_bwd_h", "gws_dense_bwd_workspace_bytes",
           "gws_adamw", "gws_grad_norm", "gws_grad_norm_workspace_bytes",
           "gws_derive_seed", "gws_status_string", "gws_version")
BENCH_EXPORTS = ("gws_copy_tiles", "gws_block_absmax", "gws_sample_bwd_tuned", "gws_sample_fwd_tuned", "gws_gemm_bf16_ride_probe", "gws_ride_plan",
                 "gws_ride_plan_layout", "gws_gemm_form", "gws_gemm_tile", "gws_gemm_stream_tile", "gws_linear_bwd_w_form", "gws_linear_bwd_w_form_rows", "gws_gated_form", "gws_dense_form", "gws_box_muller_check")
# kernels as gws_gemm_form and gws_linear_bwd_w_form name them
GEMM_STREAM, GEMM_MIDDLE, GEMM_LARGE, GEMM_LARGE_EDGE, GEMM_NARROW, GEMM_ANY_SHAPE, GEMM_STREAM_SAMPLE, GEMM_ROWS_SAMPLE, GEMM_ANY_SHAPE_SAMPLE = range(1, 10)
BWD_W_WIDE, BWD_W_NARROW, BWD_W_PIECES_64, BWD_W_PIECES_128, BWD_W_SPLIT = 1, 2, 3, 4, 16
BWD_W_PIECES_96, BWD_W_PIECES_128_128, BWD_W_PIECES_32 = 5, 6, 7
DENSE_FWD, DENSE_BWD, DENSE_SHARED = 0, 1, 10        # of gws_dense_form: the calls, and the kernel that gws_gemm_bf16 has not


class GwsError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({status_string(status)})")
        self.status = status


class _CTensor(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("w_hat", ctypes.c_void_p), ("bt", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("g", ctypes.c_void_p), ("dw", ctypes.c_void_p),
                ("dbt", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("row0", ctypes.c_int64), ("col0", ctypes.c_int64),
                ("seed", ctypes.c_uint64)]


class _CBitwidth(ctypes.Structure):
    _fields_ = [("b_init", ctypes.c_float), ("b_target", ctypes.c_float), ("lam", ctypes.c_float),
                ("layer_blocks", ctypes.c_int64)]


class _CMxOut(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("xscale", ctypes.c_void_p), ("ldc", ctypes.c_int64)]


class _CAct8(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("xscale", ctypes.c_void_p), ("ldc", ctypes.c_int64), ("lds", ctypes.c_int64)]


class _CGatedSaved(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("u", ctypes.c_void_p), ("ldg", ctypes.c_int64), ("ldu", ctypes.c_int64),
                ("g8", _CAct8), ("u8", _CAct8)]


class _CEpilogue(ctypes.Structure):
    _fields_ = [("bias", ctypes.c_void_p), ("act", ctypes.c_int), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("z", ctypes.c_void_p), ("ldz", ctypes.c_int64)]


class _CAdamWTensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("g_is_fp32", ctypes.c_int),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m8", _CAct8), ("v8", _CAct8),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("lr_scale", ctypes.c_float), ("weight_decay", ctypes.c_float), ("seed", ctypes.c_uint64)]


class _CAdamWSettings(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("step", ctypes.c_uint64), ("grad_scale", ctypes.c_void_p)]


@dataclass(slots=True)
class Act8:
    """Python-side mirror of ``gws_act8``: one-byte device tensors for the E4M3 codes [rows, columns] and the E8M0 block
    scales [rows, ceil(columns / 32)]."""
    codes: object
    xscale: object
    ldc: Optional[int] = None
    lds: Optional[int] = None


@dataclass(slots=True)
class GatedSaved:
    """Python-side mirror of ``gws_gated_saved``: G and U kept as BF16 (``g``, ``u``) or in 8 bits (``g8``, ``u8``)."""
    g: Optional[object] = None
    u: Optional[object] = None
    g8: Optional[Act8] = None
    u8: Optional[Act8] = None


@dataclass(slots=True)
class AdamWTensor:
    """Python-side mirror of ``gws_adamw_tensor``: a parameter ``p`` (fp32), its gradient (BF16 or fp32), its states ``m`` and ``v`` (both fp32, or
    both :class:`Act8`, ``v`` then holding the root) and its BF16 copy ``w``: vectors, or matrices of one leading dimension."""
    p: object
    g: object
    m: object
    v: object
    w: Optional[object] = None
    weight_decay: float = 0.0
    lr_scale: float = 1.0
    seed: int = 0


@dataclass
class MxOut:
    """Python-side mirror of ``gws_mx_out``: uint8 device tensors for element codes and E8M0 block scales."""
    codes: object
    xscale: object
    ldc: Optional[int] = None


@dataclass
class Bitwidth:
    """Python-side mirror of ``gws_bitwidth`` (paper Eq. 11 and Eq. 12), one per tensor."""
    b_init: float
    b_target: float
    lam: float = 0.0
    layer_blocks: int = 0


@dataclass
class TensorDesc:
    """Python-side mirror of ``gws_tensor``; tensor fields are torch device tensors or None."""
    rows: int
    cols: int
    seed: int
    w: Optional[object] = None
    w_hat: Optional[object] = None
    bt: Optional[object] = None
    scale: Optional[object] = None
    g: Optional[object] = None
    dw: Optional[object] = None
    dbt: Optional[object] = None
    ld: Optional[int] = None
    row0: int = 0
    col0: int = 0


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libgws.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2505_11170_amd.build` "
            "(hipcc, gfx950). There is no CPU or PyTorch fallback.")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i64, u64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int
    tp = ctypes.POINTER(_CTensor)
    L.gws_sample_fwd.argtypes = [tp, ci, ci, u64, vp]
    L.gws_sample_fwd.restype = ci
    L.gws_sample_bwd.argtypes = [tp, ci, u64, vp]
    L.gws_sample_bwd.restype = ci
    bp = ctypes.POINTER(_CBitwidth)
    L.gws_sample_fwd_bi.argtypes = [tp, ci, bp, ci, u64, vp]
    L.gws_sample_fwd_bi.restype = ci
    L.gws_sample_bwd_bi.argtypes = [tp, ci, bp, u64, vp]
    L.gws_sample_bwd_bi.restype = ci
    L.gws_sample_fwd_mx.argtypes = [tp, ctypes.POINTER(_CMxOut), ci, ci, u64, vp]
    L.gws_sample_fwd_mx.restype = ci
    L.gws_linear_fwd.argtypes = [vp, i64, i64, i64, tp, ci, ci, u64, vp, i64, vp]
    L.gws_linear_fwd.restype = ci
    L.gws_linear_fwd_mode.argtypes = [vp, i64, i64, i64, tp, ci, ci, u64, vp, i64, ci, vp]
    L.gws_linear_fwd_mode.restype = ci
    L.gws_linear_fwd_ws.argtypes = [vp, i64, i64, i64, tp, ci, ci, u64, vp, i64, vp, ctypes.c_size_t, vp]
    L.gws_linear_fwd_ws.restype = ci
    L.gws_linear_fwd_static.argtypes = [vp, i64, i64, i64, tp, ci, ci, u64, vp, i64, vp]
    L.gws_linear_fwd_static.restype = ci
    L.gws_linear_fwd_workspace_bytes.argtypes = [tp]
    L.gws_linear_fwd_workspace_bytes.restype = ctypes.c_size_t
    L.gws_gemm_bf16_sample_next.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, tp, ci, u64, vp]
    L.gws_gemm_bf16_sample_next.restype = ci
    L.gws_copy_tiles.argtypes = [tp, ci, vp]
    L.gws_copy_tiles.restype = ci
    L.gws_gemm_bf16_sample_next_n.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, tp, ci, ci, u64, vp]
    L.gws_gemm_bf16_sample_next_n.restype = ci
    L.gws_ride_plan.argtypes = [i64, i64, i64, tp, ci]
    L.gws_ride_plan.restype = ci
    L.gws_ride_plan_layout.argtypes = [i64, i64, i64, ci, tp, ci]
    L.gws_ride_plan_layout.restype = ci
    L.gws_gemm_form.argtypes = [i64, i64, i64, i64, i64, ci, ci]
    L.gws_gemm_form.restype = ci
    L.gws_gemm_tile.argtypes = [i64, i64, i64, i64, i64, ci, ci]
    L.gws_gemm_tile.restype = ci
    L.gws_gemm_stream_tile.argtypes = [i64, i64, i64, i64, i64, ci, ci]
    L.gws_gemm_stream_tile.restype = ctypes.c_uint32
    L.gws_linear_bwd_w_form.argtypes = [tp, i64, ctypes.c_size_t]
    L.gws_linear_bwd_w_form.restype = ci
    L.gws_linear_bwd_w_form_rows.argtypes = [tp, i64, ctypes.c_size_t, ci]
    L.gws_linear_bwd_w_form_rows.restype = ci
    L.gws_box_muller_check.argtypes = [u64, u64, vp, vp]
    L.gws_box_muller_check.restype = ci
    L.gws_gemm_bf16_ride_probe.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, tp, ci, u64, ci, ci, vp]
    L.gws_gemm_bf16_ride_probe.restype = ci
    L.gws_sample_fwd_tuned.argtypes = [tp, ci, ci, u64, ci, ci, vp]
    L.gws_sample_fwd_tuned.restype = ci
    L.gws_sample_bwd_tuned.argtypes = [tp, ci, u64, ci, ci, vp]
    L.gws_sample_bwd_tuned.restype = ci
    L.gws_block_absmax.argtypes = [tp, ci, vp]
    L.gws_block_absmax.restype = ci
    L.gws_linear_bwd_w.argtypes = [vp, vp, i64, i64, i64, tp, ci, u64, vp]
    L.gws_linear_bwd_w.restype = ci
    L.gws_linear_bwd_w_workspace_bytes.argtypes = [tp, i64]
    L.gws_linear_bwd_w_workspace_bytes.restype = ctypes.c_size_t
    L.gws_linear_bwd_w_ws.argtypes = [vp, vp, i64, i64, i64, tp, ci, u64, vp, ctypes.c_size_t, vp]
    L.gws_linear_bwd_w_ws.restype = ci
    L.gws_gemm_bf16.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, vp]
    L.gws_gemm_bf16.restype = ci
    L.gws_sample_fwd_basis.argtypes = [tp, ci, ci, ci, u64, vp]
    L.gws_sample_fwd_basis.restype = ci
    L.gws_sample_bwd_basis.argtypes = [tp, ci, ci, u64, vp]
    L.gws_sample_bwd_basis.restype = ci
    L.gws_noise_basis.argtypes = [vp, i64, i64, i64, i64, u64, u64, ci, vp]
    L.gws_noise_basis.restype = ci
    L.gws_noise_packed.argtypes = [vp, i64, i64, i64, i64, u64, u64, vp]
    L.gws_noise_packed.restype = ci
    L.gws_gated_form.argtypes = [ci, i64, i64, i64, i64, i64, ci, ci]
    L.gws_gated_form.restype = ci
    ap = sp = vp   # gws_act8 and gws_gated_saved, as bytes or by reference
    sz = ctypes.c_size_t
    L.gws_act8_encode.argtypes = [vp, i64, i64, i64, ap, vp]
    L.gws_act8_encode.restype = ci
    L.gws_act8_decode.argtypes = [ap, i64, i64, vp, i64, vp]
    L.gws_act8_decode.restype = ci
    L.gws_gated_fwd.argtypes = [vp, i64, i64, i64, vp, vp, i64, i64, ci, ci, vp, i64, sp, vp]
    L.gws_gated_fwd.restype = ci
    L.gws_gated_bwd.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, ci, sp, vp, vp, i64, vp, i64, vp]
    L.gws_gated_bwd.restype = ci
    L.gws_gated_bwd_h.argtypes = [vp, i64, i64, i64, ci, sp, vp, vp, i64, vp, i64, vp]
    L.gws_gated_bwd_h.restype = ci
    L.gws_gated_bwd_x.argtypes = [vp, vp, i64, i64, i64, vp, vp, i64, i64, ci, vp, i64, vp]
    L.gws_gated_bwd_x.restype = ci
    L.gws_linear_bwd_w_act8_workspace_bytes.argtypes = [tp, ci, i64]
    L.gws_linear_bwd_w_act8_workspace_bytes.restype = sz
    L.gws_linear_bwd_w_act8.argtypes = [ap, vp, i64, i64, tp, ci, u64, vp, sz, vp]
    L.gws_linear_bwd_w_act8.restype = ci
    L.gws_norm_fwd.argtypes = [vp, i64, i64, i64, ci, vp, vp, ctypes.c_float, vp, i64, vp, vp, vp]
    L.gws_norm_fwd.restype = ci
    L.gws_norm_bwd_workspace_bytes.argtypes = [i64, i64]
    L.gws_norm_bwd_workspace_bytes.restype = sz
    L.gws_norm_bwd.argtypes = [vp, i64, vp, i64, i64, i64, ci, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
    L.gws_norm_bwd.restype = ci
    L.gws_dense_fwd.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, vp, i64, vp, vp]
    L.gws_dense_fwd.restype = ci
    L.gws_dense_bwd_workspace_bytes.argtypes = [i64, i64]
    L.gws_dense_bwd_workspace_bytes.restype = sz
    L.gws_dense_bwd.argtypes = [vp, i64, i64, i64, vp, i64, i64, ci, ci, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
    L.gws_dense_bwd.restype = ci
    L.gws_dense_bwd_h.argtypes = [vp, i64, i64, i64, ci, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
    L.gws_dense_bwd_h.restype = ci
    L.gws_dense_form.argtypes = [ci, i64, i64, i64, i64, i64, ci]
    L.gws_dense_form.restype = ci
    wp = ctypes.POINTER(_CAdamWTensor)
    L.gws_adamw.argtypes = [wp, ci, vp, vp]
    L.gws_adamw.restype = ci
    L.gws_grad_norm_workspace_bytes.argtypes = [wp, ci]
    L.gws_grad_norm_workspace_bytes.restype = sz
    L.gws_grad_norm.argtypes = [wp, ci, ctypes.c_double, vp, vp, sz, vp]
    L.gws_grad_norm.restype = ci
    L.gws_derive_seed.argtypes = [u64, u64]
    L.gws_derive_seed.restype = u64
    L.gws_status_string.argtypes = [ci]
    L.gws_status_string.restype = ctypes.c_char_p
    L.gws_version.argtypes = []
    L.gws_version.restype = ci
    _lib = L
    return L


def status_string(status: int) -> str:
    try:
        return load_library().gws_status_string(int(status)).decode()
    except Exception:  # pragma: no cover
        return "?"


def _p(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_current_raw_stream = None   # torch's getters of the current device and its stream's handle, once torch is there


def _stream(stream) -> Optional[int]:
    global _current_raw_stream
    if stream is None:
        if _current_raw_stream is None:
            import torch
            torch.cuda.current_stream()   # initialises the device runtime
            device, raw = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
            _current_raw_stream = lambda: raw(device())
        return _current_raw_stream() or None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None


class PackedTensors:
    """A descriptor list already marshalled into a C array of ``gws_tensor``.

    The buffers of a training run do not move between steps, so the array can be
    built once with :func:`pack` and passed to every forward / backward call."""

    def __init__(self, arr, n, keepalive):
        self.arr, self.n, self._keepalive = arr, n, keepalive

    def __len__(self):
        return self.n


def pack(descs: Sequence[TensorDesc]) -> PackedTensors:
    return PackedTensors(_marshal(descs), len(descs), list(descs))


def _as_c(t):
    if isinstance(t, PackedTensors):
        return t.arr, t.n
    return _marshal(t), len(t)


_CTensor1 = _CTensor * 1
_pack_tensor = struct.Struct("=7Q5qQ").pack   # the fields of _CTensor in one go (field by field takes four times as long)
assert struct.calcsize("=7Q5qQ") == ctypes.sizeof(_CTensor)


def _marshal(descs: Sequence[TensorDesc]):
    if not descs:
        return _CTensor1()
    parts = []
    for d in descs:
        w, g, dw = d.w, d.g, d.dw
        ld = d.ld
        if ld is None:
            ref = w if w is not None else g if g is not None else dw
            ld = ref.stride(0) if ref is not None and ref.dim() == 2 else d.cols
        fields = (_p(w) or 0, _p(d.w_hat) or 0, _p(d.bt) or 0, _p(d.scale) or 0, _p(g) or 0, _p(dw) or 0, _p(d.dbt) or 0,
                  d.rows, d.cols, ld, d.row0, d.col0, d.seed & 0xFFFFFFFFFFFFFFFF)
        try:
            parts.append(_pack_tensor(*fields))
        except struct.error:   # not 64-bit whole numbers: as ctypes takes them, field by field (wrapped) or not at all (TypeError)
            parts.append(bytes(_CTensor(*fields)))
    if len(parts) == 1:
        return _CTensor1.from_buffer_copy(parts[0])
    return (_CTensor * len(parts)).from_buffer_copy(b"".join(parts))


def _check(rc: int, what: str):
    if rc != 0:
        raise GwsError(rc, what)


def gws_sample_fwd(t: Sequence[TensorDesc], fmt: int, step: int, stream=None) -> None:
    """Paper Eq. 3 + cast for every descriptor; writes ``w_hat`` and ``scale``."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_fwd(arr, n, int(fmt), int(step), _stream(stream)), "gws_sample_fwd")


def gws_sample_bwd(t: Sequence[TensorDesc], step: int, stream=None) -> None:
    """Paper Eq. 4 for every descriptor; writes ``dbt`` (and ``dw`` unless aliased)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_bwd(arr, n, int(step), _stream(stream)), "gws_sample_bwd")


class PackedBitwidth:
    """Bitwidth settings already marshalled into a C array of ``gws_bitwidth`` (see :func:`pack_bitwidth`)."""

    def __init__(self, arr, n):
        self.arr, self.n = arr, n

    def __len__(self):
        return self.n


def pack_bitwidth(bw: Sequence[Bitwidth]) -> PackedBitwidth:
    arr = (_CBitwidth * max(1, len(bw)))()
    for c, b in zip(arr, bw):
        c.b_init, c.b_target, c.lam, c.layer_blocks = b.b_init, b.b_target, b.lam, b.layer_blocks
    return PackedBitwidth(arr, len(bw))


def _marshal_bw(bw, n: int):
    if len(bw) != n:
        raise ValueError(f"{n} tensors but {len(bw)} bitwidth settings")
    return (bw if isinstance(bw, PackedBitwidth) else pack_bitwidth(bw)).arr


def gws_sample_fwd_bi(t: Sequence[TensorDesc], bw: Sequence[Bitwidth], fmt: int, step: int, stream=None) -> None:
    """``gws_sample_fwd`` with ``bt`` holding the internal parameter b_i of paper Eq. 11."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_fwd_bi(arr, n, _marshal_bw(bw, n), int(fmt), int(step), _stream(stream)),
           "gws_sample_fwd_bi")


def gws_sample_bwd_bi(t: Sequence[TensorDesc], bw: Sequence[Bitwidth], step: int, stream=None) -> None:
    """``gws_sample_bwd`` writing dL'/db_i (paper Eq. 11, Eq. 12) into ``dbt``; needs ``bt`` = b_i."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_bwd_bi(arr, n, _marshal_bw(bw, n), int(step), _stream(stream)), "gws_sample_bwd_bi")


class PackedMxOut:
    """MX output descriptors already marshalled into a C array of ``gws_mx_out`` (see :func:`pack_mx`)."""

    def __init__(self, arr, n, keepalive):
        self.arr, self.n, self._keepalive = arr, n, keepalive

    def __len__(self):
        return self.n


def pack_mx(outs: Sequence[MxOut]) -> PackedMxOut:
    arr = (_CMxOut * max(1, len(outs)))()
    for c, o in zip(arr, outs):
        ldc = o.ldc
        if ldc is None:
            ldc = int(o.codes.stride(0)) if o.codes is not None and o.codes.dim() == 2 else 0
        c.codes, c.xscale, c.ldc = _p(o.codes), _p(o.xscale), ldc
    return PackedMxOut(arr, len(outs), list(outs))


def gws_sample_fwd_mx(t: Sequence[TensorDesc], o: Sequence[MxOut], fmt: int, step: int, stream=None) -> None:
    """``gws_sample_fwd`` writing MX element codes and E8M0 block scales instead of ``w_hat``."""
    L = load_library()
    arr, n = _as_c(t)
    if len(o) != n:
        raise ValueError(f"{n} tensors but {len(o)} MX outputs")
    oa = (o if isinstance(o, PackedMxOut) else pack_mx(o)).arr
    _check(L.gws_sample_fwd_mx(arr, oa, n, int(fmt), int(step), _stream(stream)), "gws_sample_fwd_mx")


def gws_linear_fwd(x, w: TensorDesc, y, fmt: int, step: int, w_is_nk: bool = False, stream=None) -> None:
    """Y = X * w_hat, the weight sampled as in ``gws_sample_fwd``; the library picks the faster of its two ways."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    _check(L.gws_linear_fwd(_p(x), M, K, int(x.stride(0)), _marshal([w]), int(bool(w_is_nk)), int(fmt),
                            int(step), _p(y), int(y.stride(0)), _stream(stream)), "gws_linear_fwd")


def gws_linear_fwd_mode(x, w: TensorDesc, y, fmt: int, step: int, mode: int, w_is_nk: bool = False, stream=None) -> None:
    """``gws_linear_fwd`` with the kernel choice made by the caller (``LINEAR_*``)."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    _check(L.gws_linear_fwd_mode(_p(x), M, K, int(x.stride(0)), _marshal([w]), int(bool(w_is_nk)), int(fmt),
                                 int(step), _p(y), int(y.stride(0)), int(mode), _stream(stream)), "gws_linear_fwd_mode")


def gws_linear_fwd_workspace_bytes(w: TensorDesc) -> int:
    """Bytes of device workspace ``gws_linear_fwd_ws`` needs for this weight."""
    return int(load_library().gws_linear_fwd_workspace_bytes(_marshal([w])))


def gws_linear_fwd_ws(x, w: TensorDesc, y, fmt: int, step: int, workspace, w_is_nk: bool = False, stream=None) -> None:
    """``gws_linear_fwd`` with w_hat and scale staged in ``workspace`` (a uint8 device tensor) instead of the caller's buffers."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    _check(L.gws_linear_fwd_ws(_p(x), M, K, int(x.stride(0)), _marshal([w]), int(bool(w_is_nk)), int(fmt), int(step),
                               _p(y), int(y.stride(0)), _p(workspace), int(workspace.numel() * workspace.element_size()),
                               _stream(stream)), "gws_linear_fwd_ws")


STATIC_SCRATCH_BYTES = 32 << 20


def gws_linear_fwd_static(x, w: TensorDesc, y, fmt: int, step: int, w_is_nk: bool = False, stream=None) -> None:
    """``gws_linear_fwd_ws`` without a workspace and without any allocation: w_hat is staged in the library's own buffer."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    _check(L.gws_linear_fwd_static(_p(x), M, K, int(x.stride(0)), _marshal([w]), int(bool(w_is_nk)), int(fmt), int(step),
                                   _p(y), int(y.stride(0)), _stream(stream)), "gws_linear_fwd_static")


def _token_fields(x, dy, w: TensorDesc, w_is_nk: bool, what: str):
    """Tokens and leading dimensions of X and dY, whose rows (of one dimension or more) hold what the weight's sizes make the kernel read: the call sees
    leading dimensions alone, which columns of a wider buffer have too."""
    M, m = x.shape[0], dy.shape[0]
    K, N = (w.cols, w.rows) if w_is_nk else (w.rows, w.cols)
    if m < M or x.numel() < M * K or dy.numel() < m * N:
        raise GwsError(2, what)
    return M, x.stride()[0], dy.stride()[0]


def gws_linear_bwd_w(x, dy, w: TensorDesc, step: int, w_is_nk: bool = False, stream=None) -> None:
    """dW = X^T dY into ``w.dw`` and, when ``w.dbt`` is given, dL/db_t (paper Eq. 4) from the GEMM's epilogue."""
    L = _lib or load_library()
    _check(L.gws_linear_bwd_w(_p(x), _p(dy), *_token_fields(x, dy, w, w_is_nk, "gws_linear_bwd_w"), _marshal([w]),
                              1 if w_is_nk else 0, int(step), _stream(stream)), "gws_linear_bwd_w")


def gws_linear_bwd_w_workspace_bytes(w: TensorDesc, M: int) -> int:
    """Bytes ``gws_linear_bwd_w_ws`` would use for this weight over ``M`` tokens (0: the one-kernel form)."""
    L = load_library()
    return int(L.gws_linear_bwd_w_workspace_bytes(_marshal([w]), int(M)))


def gws_linear_bwd_w_ws(x, dy, w: TensorDesc, step: int, workspace, w_is_nk: bool = False, stream=None) -> None:
    """``gws_linear_bwd_w`` with the tokens split into parts through ``workspace`` (a device tensor, or None)."""
    L = _lib or load_library()
    nbytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(L.gws_linear_bwd_w_ws(_p(x), _p(dy), *_token_fields(x, dy, w, w_is_nk, "gws_linear_bwd_w_ws"), _marshal([w]),
                                 1 if w_is_nk else 0, int(step), _p(workspace), nbytes, _stream(stream)), "gws_linear_bwd_w_ws")


def gws_gemm_bf16(x, w, y, w_is_nk: bool = False, stream=None) -> None:
    """Plain BF16 GEMM twin of ``gws_linear_fwd`` (no sampling)."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    N = int(w.shape[0] if w_is_nk else w.shape[1])
    _check(L.gws_gemm_bf16(_p(x), M, K, int(x.stride(0)), _p(w), N, int(w.stride(0)), int(bool(w_is_nk)),
                           _p(y), int(y.stride(0)), _stream(stream)), "gws_gemm_bf16")


def gws_gemm_bf16_sample_next(x, w, y, nxt: Optional[TensorDesc], fmt: int, step: int, w_is_nk: bool = False, stream=None) -> None:
    """``gws_gemm_bf16`` with ``gws_sample_fwd([nxt], fmt, step)`` riding along in the same launch where that pays."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    N = int(w.shape[0] if w_is_nk else w.shape[1])
    arr = None if nxt is None else _marshal([nxt])
    _check(L.gws_gemm_bf16_sample_next(_p(x), M, K, int(x.stride(0)), _p(w), N, int(w.stride(0)), int(bool(w_is_nk)),
                                       _p(y), int(y.stride(0)), arr, int(fmt), int(step), _stream(stream)),
           "gws_gemm_bf16_sample_next")


def gws_gemm_bf16_sample_next_n(x, w, y, nxt, fmt: int, step: int, w_is_nk: bool = False, stream=None) -> None:
    """``gws_gemm_bf16`` with ``gws_sample_fwd(nxt, fmt, step)`` of a list of weights riding along where that pays."""
    L = load_library()
    M, K = int(x.shape[0]), int(x.shape[1])
    N = int(w.shape[0] if w_is_nk else w.shape[1])
    arr, n = _as_c(nxt)
    _check(L.gws_gemm_bf16_sample_next_n(_p(x), M, K, int(x.stride(0)), _p(w), N, int(w.stride(0)), int(bool(w_is_nk)),
                                         _p(y), int(y.stride(0)), arr, n, int(fmt), int(step), _stream(stream)),
           "gws_gemm_bf16_sample_next_n")


def gws_ride_plan(M: int, K: int, N: int, nxt, w_is_nk: bool = False) -> int:
    """How many of ``nxt`` would ride in the launch of an M x K x N GEMM (a measurement aid)."""
    arr, n = _as_c(nxt)
    return int(load_library().gws_ride_plan_layout(int(M), int(K), int(N), int(bool(w_is_nk)), arr, n))


def gws_gemm_form(M: int, K: int, N: int, w_is_nk: bool = False, sampled: int = 0, ldx: Optional[int] = None, ldw: Optional[int] = None) -> int:
    """The kernel (``GEMM_*``) of ``gws_gemm_bf16`` (``sampled`` 0), of ``LINEAR_IN_OPERAND`` (1) or of ``gws_linear_fwd`` with w_hat (2)."""
    return int(load_library().gws_gemm_form(int(M), int(K), K if ldx is None else int(ldx), int(N), (K if w_is_nk else N) if ldw is None else int(ldw),
                                            int(bool(w_is_nk)), int(sampled)))


def gws_gemm_tile(M: int, K: int, N: int, w_is_nk: bool = False, sampled: int = 0, ldx: Optional[int] = None, ldw: Optional[int] = None) -> tuple:
    """Rows and columns of Y that a workgroup of that kernel makes; (0, 0) for sizes that the call refuses."""
    t = int(load_library().gws_gemm_tile(int(M), int(K), K if ldx is None else int(ldx), int(N), (K if w_is_nk else N) if ldw is None else int(ldw),
                                         int(bool(w_is_nk)), int(sampled)))
    return t >> 16, t & 0xFFFF


def gws_gemm_stream_tile(M: int, K: int, N: int, w_is_nk: bool = False, ldx: Optional[int] = None, ldw: Optional[int] = None,
                         sampled: int = 0) -> tuple:
    """Of the call that ``gws_gemm_form`` with these arguments names, by ``GEMM_STREAM``: rows and columns that a workgroup stores, workgroups a
    tile that only fetch the weight into the L2s, whether each XCD takes a contiguous part of the tiles; zeros for another kernel."""
    t = int(load_library().gws_gemm_stream_tile(int(M), int(K), K if ldx is None else int(ldx), int(N), (K if w_is_nk else N) if ldw is None else int(ldw),
                                                int(bool(w_is_nk)), int(sampled)))
    return t >> 24, t >> 16 & 0xFF, t >> 8 & 0xFF, t & 0xFF


def gws_linear_bwd_w_form(w: TensorDesc, M: int, workspace_bytes: int = 0, on_lines: bool = True) -> int:
    """The form (``BWD_W_*``) that ``gws_linear_bwd_w_ws`` takes with that much workspace; ``BWD_W_SPLIT`` plus the number of parts.
    ``on_lines``: every row of X, dY and dW starts on a 128-byte line, as contiguous ones do."""
    return int(load_library().gws_linear_bwd_w_form_rows(_marshal([w]), int(M), int(workspace_bytes), int(on_lines)))


def gws_gemm_bf16_ride_probe(x, w, y, nxt: TensorDesc, fmt: int, step: int, extra_workgroups: int, rider: int = 1,
                             w_is_nk: bool = False, stream=None) -> None:
    """``gws_gemm_bf16_sample_next`` with the riding forced (a measurement aid); ``x=None`` launches the riders alone."""
    L = load_library()
    if x is None:
        M = K = N = ldx = ldw = ldy = 0
    else:
        M, K = int(x.shape[0]), int(x.shape[1])
        N = int(w.shape[0] if w_is_nk else w.shape[1])
        ldx, ldw, ldy = int(x.stride(0)), int(w.stride(0)), int(y.stride(0))
    _check(L.gws_gemm_bf16_ride_probe(_p(x), M, K, ldx, _p(w), N, ldw, int(bool(w_is_nk)), _p(y), ldy, _marshal([nxt]),
                                      int(fmt), int(step), int(extra_workgroups), int(rider), _stream(stream)),
           "gws_gemm_bf16_ride_probe")


def gws_copy_tiles(t: Sequence[TensorDesc], stream=None) -> None:
    """Copy ``w`` to ``w_hat`` with the forward pass's access pattern (a measurement aid)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_copy_tiles(arr, n, _stream(stream)), "gws_copy_tiles")


def gws_sample_bwd_tuned(t: Sequence[TensorDesc], step: int, variant: int = -1, per_x: int = 0, stream=None) -> None:
    """``gws_sample_bwd`` with the kernel variant and the column tiles per workgroup chosen by the caller (a measurement aid)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_bwd_tuned(arr, n, int(step), int(variant), int(per_x), _stream(stream)), "gws_sample_bwd_tuned")


def gws_sample_fwd_tuned(t: Sequence[TensorDesc], fmt: int, step: int, variant: int = -1, per_x: int = 0, stream=None) -> None:
    """``gws_sample_fwd`` with the kernel variant and the column tiles per workgroup chosen by the caller (a measurement aid)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_fwd_tuned(arr, n, int(fmt), int(step), int(variant), int(per_x), _stream(stream)), "gws_sample_fwd_tuned")


def gws_block_absmax(t: Sequence[TensorDesc], stream=None) -> None:
    """``scale`` := max|w| per 32x32 block (step one of paper Eq. 3; also the read-only ceiling measurement)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_block_absmax(arr, n, _stream(stream)), "gws_block_absmax")


# A kernel reads BF16 rows, or bytes, in memory order: other types and spread columns are told here, where the tensors still say so.  The calls
# compare in line (a function for every tensor takes as long as the call) and come here only for the message, and once for torch's types.
_bf16, _one_byte = None, frozenset()


def _check_plain(*matrices) -> None:
    global _bf16
    if _bf16 is None:
        import torch
        _bf16 = torch.bfloat16
    for t in matrices:
        if t.dtype is not _bf16 or (t.stride()[1] != 1 and t.shape[1] > 1):
            raise ValueError(f"a matrix is BF16 with its columns next to each other, not {t.dtype} of shape {list(t.shape)} and strides {list(t.stride())}")


def _check_bytes(*matrices) -> None:
    global _one_byte
    for t in matrices:
        if t.element_size() != 1 or (t.stride()[1] != 1 and t.shape[1] > 1):
            raise ValueError(f"codes and scales are of one byte and next to each other, not {t.dtype} of shape {list(t.shape)} and strides {list(t.stride())}")
        _one_byte |= {t.dtype}


# (stride() whole: half the time of stride(0), which takes its argument apart)
_pack_act8 = struct.Struct("=2Q2q").pack
_pack_saved = struct.Struct("=2Q2q2Q2q2Q2q").pack   # the fields in one go, passed as bytes (building the structures takes as long as the call)
assert struct.calcsize("=2Q2q") == ctypes.sizeof(_CAct8) and struct.calcsize("=2Q2q2Q2q2Q2q") == ctypes.sizeof(_CGatedSaved)


def _act8_fields(a: Act8, rows: int, cols: int):
    c, s, ldc, lds = a.codes, a.xscale, a.ldc, a.lds
    if c.shape != (rows, cols) or s.shape != (rows, -(-cols // 32)):
        raise ValueError(f"[{rows}, {cols}] in 8 bits has codes of that shape and scales [{rows}, {-(-cols // 32)}], not {list(c.shape)} and {list(s.shape)}")
    (cs, c1), (ss, s1) = c.stride(), s.stride()
    if c1 != 1 or s1 != 1 or c.dtype not in _one_byte or s.dtype not in _one_byte:
        _check_bytes(c, s)
    return c.data_ptr(), s.data_ptr(), cs if ldc is None else ldc, ss if lds is None else lds


def _marshal_saved(s: Optional[GatedSaved], rows: int, cols: int):
    if s is None:
        return None
    g, u, g8, u8 = s.g, s.u, s.g8, s.u8
    if g8 is None and u8 is None and g is not None and u is not None:
        if g.shape != (rows, cols) or u.shape != (rows, cols):
            raise ValueError(f"a kept G or U has shape {list(g.shape)} or {list(u.shape)}, not [{rows}, {cols}]")
        (ldg, g1), (ldu, u1) = g.stride(), u.stride()
        if not (g1 == u1 == 1 and g.dtype is u.dtype is _bf16):
            _check_plain(g, u)
        return _pack_saved(g.data_ptr(), u.data_ptr(), ldg, ldu, 0, 0, 0, 0, 0, 0, 0, 0)
    if g is None and u is None and g8 is not None and u8 is not None:
        return _pack_saved(0, 0, 0, 0, *_act8_fields(g8, rows, cols), *_act8_fields(u8, rows, cols))
    raise ValueError("G and U are kept both as BF16 (g, u) or both in 8 bits (g8, u8)")


def gws_act8_encode(x, o: Act8, stream=None) -> None:
    """BF16 ``x`` [rows, columns] to E4M3 codes and a scale for every 32 of a row."""
    (M, C), (ldx, x1) = x.shape, x.stride()
    if x1 != 1 or x.dtype is not _bf16:
        _check_plain(x)
    _check((_lib or load_library()).gws_act8_encode(x.data_ptr(), M, C, ldx, _pack_act8(*_act8_fields(o, M, C)), _stream(stream)), "gws_act8_encode")


def gws_act8_decode(a: Act8, x, stream=None) -> None:
    """The values of such codes into BF16 ``x``; exact."""
    (M, C), (ldx, x1) = x.shape, x.stride()
    if x1 != 1 or x.dtype is not _bf16:
        _check_plain(x)
    _check((_lib or load_library()).gws_act8_decode(_pack_act8(*_act8_fields(a, M, C)), M, C, x.data_ptr(), ldx, _stream(stream)), "gws_act8_decode")


def gws_gated_fwd(x, wg, wu, h, act: int = ACT_SILU, saved: Optional[GatedSaved] = None, w_is_nk: bool = False, stream=None) -> None:
    """H = a(X Wg) * (X Wu) by elements in one kernel; ``saved`` receives G and U for the backward pass."""
    (M, K), size = x.shape, wg.shape
    (ldx, x1), (ldw, g1), (ldwu, u1), (ldh, h1) = x.stride(), wg.stride(), wu.stride(), h.stride()
    F, Kw = size if w_is_nk else (size[1], size[0])
    if Kw != K or wu.shape != size or h.shape != (M, F):
        raise ValueError(f"X {list(x.shape)}, Wg {list(size)}, Wu {list(wu.shape)} and H {list(h.shape)} do not fit together")
    if not (x1 == g1 == u1 == h1 == 1 and x.dtype is wg.dtype is wu.dtype is h.dtype is _bf16):
        _check_plain(x, wg, wu, h)
    if ldwu != ldw:
        raise ValueError(f"leading dimensions of Wg and Wu differ: {ldw} and {ldwu}")
    _check((_lib or load_library()).gws_gated_fwd(x.data_ptr(), M, K, ldx, wg.data_ptr(), wu.data_ptr(), F, ldw, 1 if w_is_nk else 0, act,
                                                  h.data_ptr(), ldh, _marshal_saved(saved, M, F), _stream(stream)), "gws_gated_fwd")


def _gradient_fields(dg, du, h, M, F):
    """dG, dU, their leading dimension, H and its."""
    size, (ldd, g1), (lddu, u1) = (M, F), dg.stride(), du.stride()
    ldh, h1 = (0, 1) if h is None else h.stride()
    if dg.shape != size or du.shape != size or (h is not None and h.shape != size):
        raise ValueError(f"dG, dU and H have shape [{M}, {F}]")
    if not (g1 == u1 == h1 == 1 and dg.dtype is du.dtype is _bf16 and (h is None or h.dtype is _bf16)):
        _check_plain(*((dg, du) if h is None else (dg, du, h)))
    if lddu != ldd:
        raise ValueError(f"leading dimensions of dG and dU differ: {ldd} and {lddu}")
    return dg.data_ptr(), du.data_ptr(), ldd, None if h is None else h.data_ptr(), ldh


def gws_gated_bwd(dy, wd, saved: GatedSaved, dg, du, act: int = ACT_SILU, h=None, w_is_nk: bool = False, stream=None) -> None:
    """dG and dU (and H again) from the gradient of Y = H Wd and the kept G and U; dH = dY Wd^T stays in the kernel."""
    (M, D), size = dy.shape, wd.shape
    (ldy, y1), (ldw, w1) = dy.stride(), wd.stride()
    F, Dw = (size[1], size[0]) if w_is_nk else size
    if Dw != D:
        raise ValueError(f"dY {list(dy.shape)} and Wd {list(size)} do not fit together")
    if not (y1 == w1 == 1 and dy.dtype is wd.dtype is _bf16):
        _check_plain(dy, wd)
    _check((_lib or load_library()).gws_gated_bwd(dy.data_ptr(), M, D, ldy, wd.data_ptr(), F, ldw, 1 if w_is_nk else 0, act,
                                                  _marshal_saved(saved, M, F), *_gradient_fields(dg, du, h, M, F), _stream(stream)), "gws_gated_bwd")


def gws_gated_bwd_h(dh, saved: GatedSaved, dg, du, act: int = ACT_SILU, h=None, stream=None) -> None:
    """``gws_gated_bwd`` from a given dH."""
    (M, F), (ldh, h1) = dh.shape, dh.stride()
    if h1 != 1 or dh.dtype is not _bf16:
        _check_plain(dh)
    _check((_lib or load_library()).gws_gated_bwd_h(dh.data_ptr(), M, F, ldh, act, _marshal_saved(saved, M, F),
                                                    *_gradient_fields(dg, du, h, M, F), _stream(stream)), "gws_gated_bwd_h")


def gws_gated_bwd_x(dg, du, wg, wu, dx, w_is_nk: bool = False, stream=None) -> None:
    """dX = dG Wg^T + dU Wu^T in one sum; ``w_is_nk`` as in ``gws_gated_fwd``."""
    (M, F), size = dg.shape, wg.shape
    (ldd, d1), (lddu, e1), (ldw, g1), (ldwu, u1), (ldx, x1) = dg.stride(), du.stride(), wg.stride(), wu.stride(), dx.stride()
    K, Fw = (size[1], size[0]) if w_is_nk else size
    if Fw != F or wu.shape != size or du.shape != (M, F) or dx.shape != (M, K):
        raise ValueError(f"dG {list(dg.shape)}, dU {list(du.shape)}, Wg {list(size)}, Wu {list(wu.shape)} and dX {list(dx.shape)} do not fit together")
    if not (d1 == e1 == g1 == u1 == x1 == 1 and dg.dtype is du.dtype is wg.dtype is wu.dtype is dx.dtype is _bf16):
        _check_plain(dg, du, wg, wu, dx)
    if ldwu != ldw or lddu != ldd:
        raise ValueError(f"leading dimensions differ: dG and dU {ldd} and {lddu}, Wg and Wu {ldw} and {ldwu}")
    _check((_lib or load_library()).gws_gated_bwd_x(dg.data_ptr(), du.data_ptr(), M, F, ldd, wg.data_ptr(), wu.data_ptr(), K, ldw, 1 if w_is_nk else 0,
                                                    dx.data_ptr(), ldx, _stream(stream)), "gws_gated_bwd_x")


def gws_gated_form(op: int, M: int, K: int, F: int, w_is_nk: bool = False, kept: int = 0, lda: Optional[int] = None, ldw: Optional[int] = None) -> tuple:
    """The kernel (``GATED_*``) of a call (``GATED_FWD``, ``GATED_BWD`` with K columns of dY, ``GATED_BWD_X``) and, of ``GATED_STREAM``, its tile in
    units of 16 rows and columns; ``kept``: 0 nothing, 1 BF16, 2 in 8 bits.  0 for sizes that the call refuses.  A call of two launches: of the first
    (``gws_gated_forms`` has both)."""
    return gws_gated_forms(op, M, K, F, w_is_nk, kept, lda, ldw)[0]


def gws_gated_forms(op: int, M: int, K: int, F: int, w_is_nk: bool = False, kept: int = 0, lda: Optional[int] = None, ldw: Optional[int] = None) -> tuple:
    """``gws_gated_form`` of the first launch, the kernel of the second (0: there is none), and whether the launches share the rows rather than the columns."""
    f = _gated_form(op, M, K, F, w_is_nk, kept, lda, ldw)
    return (f & 0xFF, f >> 16 & 0xFF, f >> 8 & 0xFF), f >> 24 & 0xF, bool(f >> 28 & 1)


def gws_gated_past_caches(op: int, M: int, K: int, F: int, w_is_nk: bool = False, kept: int = 0, lda: Optional[int] = None, ldw: Optional[int] = None) -> bool:
    """Whether the 128 x 128 and 256 x 256 tiles of such a call store H, or dG, dU and H, past the caches."""
    return bool(_gated_form(op, M, K, F, w_is_nk, kept, lda, ldw) >> 29 & 1)


def _gated_form(op, M, K, F, w_is_nk, kept, lda, ldw) -> int:
    wide = op == GATED_BWD
    return int(load_library().gws_gated_form(op, M, K, F, (F if op == GATED_BWD_X else K) if lda is None else lda,
                                             (F if w_is_nk == wide else K) if ldw is None else ldw, int(bool(w_is_nk)), kept))


def gws_linear_bwd_w_act8_workspace_bytes(w: TensorDesc, M: int, w_is_nk: bool = False) -> int:
    """Bytes of workspace that ``gws_linear_bwd_w_act8`` can use for this weight over ``M`` tokens."""
    return int(load_library().gws_linear_bwd_w_act8_workspace_bytes(_marshal([w]), int(bool(w_is_nk)), int(M)))


def gws_linear_bwd_w_act8(x: Act8, dy, w: TensorDesc, step: int, workspace, w_is_nk: bool = False, stream=None) -> None:
    """``gws_linear_bwd_w_ws`` with the linear's input kept in 8 bits."""
    (M, Ny), (ldy, y1) = dy.shape, dy.stride()
    K, N = (w.cols, w.rows) if w_is_nk else (w.rows, w.cols)
    if y1 != 1 or dy.dtype is not _bf16:
        _check_plain(dy)
    # the call itself sees leading dimensions alone, which columns of a wider buffer have too
    if Ny != N or (w.dw is not None and w.dw.shape != (w.rows, w.cols)):
        raise ValueError(f"dY {list(dy.shape)} and dW {None if w.dw is None else list(w.dw.shape)} do not fit a weight of {w.rows} x {w.cols} with N = {N}")
    nbytes = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(load_library().gws_linear_bwd_w_act8(_pack_act8(*_act8_fields(x, M, K)), _p(dy), M, ldy, _marshal([w]), 1 if w_is_nk else 0, int(step), _p(workspace),
                                                nbytes, _stream(stream)), "gws_linear_bwd_w_act8")


# The calls below look at their tensors in line (each attribute of a tensor takes as long as a function's call) and come to these for what is out of the ordinary:
# a message, or one row or column, whose stride says nothing.
_fp32 = None


def _look_at_matrix(t, shape, device: int):
    """Address and leading dimension of a BF16 matrix, or what is wrong with it."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"a matrix has shape {list(t.shape)}, not {list(shape)}")
    if t.dtype is not _bf16 or (t.stride()[1] != 1 and shape[1] > 1):
        _check_plain(t)
    _check_device(device, t)
    return t.data_ptr(), t.stride()[0] if shape[0] > 1 else -(-shape[1] // 8) * 8


def _matrix(t, size, device: int):
    if t is None:
        return None, 0
    ld, one = t.stride()
    if t.shape != size or one != 1 or t.dtype is not _bf16 or t.get_device() != device:
        return _look_at_matrix(t, size, device)
    return t.data_ptr(), ld if size[0] != 1 else -(-size[1] // 8) * 8   # one row's stride says nothing


def _look_at_vector(t, n: int, device: int):
    global _fp32
    if _fp32 is None:
        import torch
        _fp32 = torch.float32
    if t.dtype is not _fp32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"a vector here is fp32 of {n} elements next to each other, not {t.dtype} of shape {list(t.shape)} and strides {list(t.stride())}")
    _check_device(device, t)
    return t.data_ptr()


def _vector(t, n: int, device: int):
    if t is None:
        return None
    if t.dtype is not _fp32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        return _look_at_vector(t, n, device)
    return t.data_ptr()


def _bytes_of(workspace, device: int):
    if workspace is None:
        return None, 0
    if workspace.get_device() != device or not workspace.is_contiguous():
        _check_device(device, workspace)
        raise ValueError("a workspace is contiguous")
    return workspace.data_ptr(), workspace.nbytes


def _check_device(device: int, *tensors) -> None:
    for t in tensors:
        if t.get_device() != device:
            raise ValueError(f"the tensors of a call are on one device, not on {device} and {t.get_device()} (-1: host memory)")


_get_device = _get_raw_stream = None   # torch's current device and its stream's handle, once torch is there


def _stream_of(device: int, stream):
    """The stream of a call on tensors of `device`, which has to be the current one: a launch goes to the current device's stream."""
    global _get_device, _get_raw_stream
    if _get_device is None:
        import torch
        if device >= 0:
            torch.cuda.current_stream()   # initialises the device runtime
        _get_device, _get_raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    if device < 0 or _get_device() != device or (stream is not None and not isinstance(stream, int) and stream.device_index != device):
        raise ValueError(f"the tensors are on device {device} (-1: host memory), which is not the current device or the stream's")
    return (_get_raw_stream(device) or None) if stream is None else _stream(stream)


def gws_norm_fwd(x, y, kind: int = NORM_LAYER, gamma=None, beta=None, eps: float = 1e-5, mean=None, rstd=None, stream=None) -> None:
    """Layer norm or root-mean-square norm of the rows of ``x`` into ``y``; ``mean`` and ``rstd`` (fp32, one a row) receive what the backward pass needs."""
    size, on = x.shape, x.get_device()
    M, C = size
    (px, ldx), (py, ldy) = _matrix(x, size, on), _matrix(y, size, on)
    _check((_lib or load_library()).gws_norm_fwd(px, M, C, ldx, kind, _vector(gamma, C, on), _vector(beta, C, on), eps, py, ldy, _vector(mean, M, on),
                                                 _vector(rstd, M, on), _stream_of(on, stream)), "gws_norm_fwd")


def gws_norm_bwd_workspace_bytes(M: int, C: int) -> int:
    """Bytes of workspace that ``gws_norm_bwd`` needs for dgamma, dbeta or rows of more than 16384 columns."""
    return int(load_library().gws_norm_bwd_workspace_bytes(M, C))


def gws_norm_bwd(dy, x, dx, rstd, kind: int = NORM_LAYER, mean=None, gamma=None, residual=None, dgamma=None, dbeta=None, workspace=None, stream=None) -> None:
    """dX of the norm, plus ``residual`` (a gradient that comes past it), with dgamma and dbeta; ``mean`` and ``rstd`` as ``gws_norm_fwd`` kept them."""
    size, on = x.shape, x.get_device()
    M, C = size
    (pdy, lddy), (px, ldx), (pr, ldr), (pdx, lddx) = _matrix(dy, size, on), _matrix(x, size, on), _matrix(residual, size, on), _matrix(dx, size, on)
    _check((_lib or load_library()).gws_norm_bwd(pdy, lddy, px, M, C, ldx, kind, _vector(gamma, C, on), _vector(mean, M, on), _vector(rstd, M, on), pr, ldr, pdx, lddx,
                                                 _vector(dgamma, C, on), _vector(dbeta, C, on), *_bytes_of(workspace, on), _stream_of(on, stream)), "gws_norm_bwd")


_pack_epilogue = struct.Struct("=Qi4xQqQq").pack
assert struct.calcsize("=Qi4xQqQq") == ctypes.sizeof(_CEpilogue)


def gws_dense_fwd(x, w, y, bias=None, act: int = ACT_NONE, residual=None, z=None, w_is_nk: bool = False, stream=None) -> None:
    """Y = a(X W + b) + R in one kernel; ``z`` receives X W + b for the backward pass."""
    xs, ws, on = x.shape, w.shape, x.get_device()
    M, K = xs
    N, Kw = ws if w_is_nk else (ws[1], ws[0])
    if Kw != K:
        raise ValueError(f"X {list(xs)} and W {list(ws)} do not fit together")
    ys = (M, N)
    (px, ldx), (pw, ldw), (py, ldy), (pr, ldr), (pz, ldz) = _matrix(x, xs, on), _matrix(w, ws, on), _matrix(y, ys, on), _matrix(residual, ys, on), _matrix(z, ys, on)
    _check((_lib or load_library()).gws_dense_fwd(px, M, K, ldx, pw, N, ldw, 1 if w_is_nk else 0, py, ldy,
                                                  _pack_epilogue(_vector(bias, N, on) or 0, act, pr or 0, ldr, pz or 0, ldz), _stream_of(on, stream)), "gws_dense_fwd")


def gws_dense_bwd_workspace_bytes(M: int, F: int) -> int:
    """Bytes of workspace that ``gws_dense_bwd`` and ``gws_dense_bwd_h`` need for ``dbias``."""
    return int(load_library().gws_dense_bwd_workspace_bytes(M, F))


def gws_dense_bwd(dy, wd, z, dz, act: int = ACT_NONE, h=None, dbias=None, workspace=None, w_is_nk: bool = False, stream=None) -> None:
    """dZ (and H = a(Z) again, and the bias gradient) from the gradient of Y = H Wd and the kept Z; dH = dY Wd^T stays in the kernel."""
    ys, ws, on = dy.shape, wd.shape, dy.get_device()
    M, D = ys
    F, Dw = (ws[1], ws[0]) if w_is_nk else ws
    if Dw != D:
        raise ValueError(f"dY {list(ys)} and Wd {list(ws)} do not fit together")
    zs = (M, F)
    (pdy, lddy), (pw, ldw), (pz, ldz), (pd, ldd), (ph, ldh) = _matrix(dy, ys, on), _matrix(wd, ws, on), _matrix(z, zs, on), _matrix(dz, zs, on), _matrix(h, zs, on)
    _check((_lib or load_library()).gws_dense_bwd(pdy, M, D, lddy, pw, F, ldw, 1 if w_is_nk else 0, act, pz, ldz, pd, ldd, ph, ldh, _vector(dbias, F, on),
                                                  *_bytes_of(workspace, on), _stream_of(on, stream)), "gws_dense_bwd")


def gws_dense_bwd_h(dh, z, dz, act: int = ACT_NONE, h=None, dbias=None, workspace=None, stream=None) -> None:
    """``gws_dense_bwd`` from a given dH; with ``ACT_NONE`` ``z`` and ``dz`` may be None, which leaves the bias gradient alone."""
    size, on = dh.shape, dh.get_device()
    M, F = size
    (pdy, lddy), (pz, ldz), (pd, ldd), (ph, ldh) = _matrix(dh, size, on), _matrix(z, size, on), _matrix(dz, size, on), _matrix(h, size, on)
    _check((_lib or load_library()).gws_dense_bwd_h(pdy, M, F, lddy, act, pz, ldz, pd, ldd, ph, ldh, _vector(dbias, F, on), *_bytes_of(workspace, on),
                                                    _stream_of(on, stream)), "gws_dense_bwd_h")


def gws_dense_form(op: int, M: int, K: int, N: int, w_is_nk: bool = False, ldx: Optional[int] = None, ldw: Optional[int] = None) -> int:
    """The kernel (``GEMM_*``, ``DENSE_SHARED``) of ``gws_dense_fwd`` (``DENSE_FWD``) or ``gws_dense_bwd`` (``DENSE_BWD``: K columns of dY, N of dZ)."""
    along = bool(w_is_nk) == (op == DENSE_FWD)
    return int(load_library().gws_dense_form(op, M, K, N, K if ldx is None else ldx, (K if along else N) if ldw is None else ldw, int(bool(w_is_nk))))


class PackedAdamW:
    """A list of parameters already marshalled into a C array of ``gws_adamw_tensor`` (see :func:`pack_adamw`)."""

    def __init__(self, arr, n, keepalive, device):
        self.arr, self.n, self._keepalive, self.device = arr, n, keepalive, device

    def __len__(self):
        return self.n


def pack_adamw(tensors: Sequence[AdamWTensor]) -> PackedAdamW:
    """The buffers of a training run do not move between steps, so the array can be built once and passed to every call."""
    import torch

    arr = (_CAdamWTensor * max(1, len(tensors)))()
    on = tensors[0].p.get_device() if len(tensors) else None
    for c, t in zip(arr, tensors):
        shape = t.p.shape
        if len(shape) not in (1, 2):
            raise ValueError(f"a parameter is a vector or a matrix, not of shape {list(shape)}")
        rows, cols = shape if len(shape) == 2 else (1, shape[0])

        def place(name, x, dtypes, want=shape):
            if x.shape != want or x.dtype not in dtypes or (want[-1] > 1 and x.stride()[-1] != 1):
                raise ValueError(f"{name} is {' or '.join(str(d) for d in dtypes)} of shape {list(want)} with its columns next to each other, not {x.dtype} of "
                                 f"shape {list(x.shape)} and strides {list(x.stride())}")
            _check_device(on, x)
            return x.data_ptr(), x.stride()[0] if len(want) == 2 and rows > 1 else None

        found = []   # leading dimensions
        c.p, ld = place("p", t.p, (torch.float32,))
        found.append(ld)
        c.g, ld = place("g", t.g, (torch.bfloat16, torch.float32))
        found.append(ld)
        c.g_is_fp32 = int(t.g.dtype is torch.float32)
        if t.w is not None:
            c.w, ld = place("w", t.w, (torch.bfloat16,))
            found.append(ld)
        if isinstance(t.m, Act8) != isinstance(t.v, Act8):
            raise ValueError("m and v are held both in 32 bits or both in 8")
        if isinstance(t.m, Act8):
            one_byte = (torch.uint8, torch.int8, torch.float8_e4m3fn, torch.float8_e8m0fnu)
            blocks = shape[:-1] + (-(-cols // 32),)
            for name, s, to in (("m", t.m, c.m8), ("v", t.v, c.v8)):
                to.codes, ld = place(f"{name}'s codes", s.codes, one_byte)
                found.append(ld if s.ldc is None else s.ldc)
                to.xscale, lds = place(f"{name}'s scales", s.xscale, one_byte, blocks)
                to.lds = s.lds if s.lds is not None else lds if lds is not None else blocks[-1]
        else:
            c.m, ld = place("m", t.m, (torch.float32,))
            found.append(ld)
            c.v, ld = place("v", t.v, (torch.float32,))
            found.append(ld)
        lds = {x for x in found if x is not None} or {-(-cols // 8) * 8}   # one row: any
        if len(lds) != 1:
            raise ValueError(f"the arrays of a parameter have one leading dimension, not {sorted(lds)}")
        c.rows, c.cols, c.ld = rows, cols, lds.pop()
        c.m8.ldc = c.v8.ldc = c.ld
        c.lr_scale, c.weight_decay, c.seed = t.lr_scale, t.weight_decay, t.seed & (2 ** 64 - 1)
    return PackedAdamW(arr, len(tensors), list(tensors), on)


_pack_settings = struct.Struct("=4d2Q").pack
assert struct.calcsize("=4d2Q") == ctypes.sizeof(_CAdamWSettings)


def gws_adamw(t, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, grad_scale=None, stream=None) -> None:
    """One AdamW step (``step`` = 1, 2, ...) over a list of :class:`AdamWTensor`, or :func:`pack_adamw`'s array; ``grad_scale``: a device fp32 number that
    the gradients are multiplied by, as ``gws_grad_norm`` leaves it (not finite: the step is left out)."""
    if not isinstance(t, PackedAdamW):
        t = pack_adamw(t)
    if not 0 < step < 2 ** 64:
        raise ValueError(f"steps are 1, 2, ..., not {step}")
    n, on = t.n, t.device
    _check((_lib or load_library()).gws_adamw(t.arr, n, _pack_settings(lr, beta1, beta2, eps, step, _vector(grad_scale, 1, on) or 0 if n else 0),
                                              _stream_of(on, stream) if n else None), "gws_adamw")


def gws_grad_norm_workspace_bytes(t) -> int:
    """Bytes of workspace that ``gws_grad_norm`` needs for these tensors."""
    t = t if isinstance(t, PackedAdamW) else pack_adamw(t)
    return int(load_library().gws_grad_norm_workspace_bytes(t.arr, t.n))


def gws_grad_norm(t, out, workspace, max_norm: float = 0.0, stream=None) -> None:
    """``out`` (fp32 [2]): the norm of all gradients, and the factor that takes it down to ``max_norm`` where it is larger."""
    if not isinstance(t, PackedAdamW):
        t = pack_adamw(t)
    on = t.device if t.n else out.get_device()
    _check((_lib or load_library()).gws_grad_norm(t.arr, t.n, max_norm, _vector(out, 2, on), *_bytes_of(workspace, on), _stream_of(on, stream)), "gws_grad_norm")


def gws_sample_fwd_basis(t: Sequence[TensorDesc], basis: int, fmt: int, step: int, stream=None) -> None:
    """``gws_sample_fwd`` with R drawn from a comparison basis (``BASIS_*``; paper Sec. 4)."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_fwd_basis(arr, n, int(basis), int(fmt), int(step), _stream(stream)), "gws_sample_fwd_basis")


def gws_sample_bwd_basis(t: Sequence[TensorDesc], basis: int, step: int, stream=None) -> None:
    """``gws_sample_bwd`` with R drawn from a comparison basis."""
    L = load_library()
    arr, n = _as_c(t)
    _check(L.gws_sample_bwd_basis(arr, n, int(basis), int(step), _stream(stream)), "gws_sample_bwd_basis")


def gws_noise_basis(out, rows: int, cols: int, seed: int, step: int, basis: int, row0: int = 0, col0: int = 0,
                    stream=None) -> None:
    """R of a comparison basis as BF16 values into ``out`` [rows, cols]."""
    L = load_library()
    _check(L.gws_noise_basis(_p(out), rows, cols, row0, col0, seed & (2 ** 64 - 1), int(step), int(basis),
                             _stream(stream)), "gws_noise_basis")


def gws_box_muller_check(out, first: int = 0, n: int = 2 ** 32, stream=None) -> None:
    """Both ways to R of the Box-Muller basis over ``n`` words of noise, compared; ``out``: three int64 on the device, added to."""
    _check(load_library().gws_box_muller_check(int(first), int(n), _p(out), _stream(stream)), "gws_box_muller_check")


def gws_noise_packed(out, rows: int, cols: int, seed: int, step: int, row0: int = 0, col0: int = 0,
                     stream=None) -> None:
    """Packed sign-magnitude noise codes, 8 per 32-bit word (paper Sec. 3.4)."""
    L = load_library()
    _check(L.gws_noise_packed(_p(out), rows, cols, row0, col0, seed & (2 ** 64 - 1), int(step),
                              _stream(stream)), "gws_noise_packed")


def gws_derive_seed(user_seed: int, tensor_id: int) -> int:
    return int(load_library().gws_derive_seed(user_seed & (2 ** 64 - 1), tensor_id & (2 ** 64 - 1)))


derive_seed = gws_derive_seed
