"""ctypes binding over the HDQT C-ABI library (include/hdqt.h).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  PyTorch supplies device memory and the current stream.  There is no
CPU fallback: if the library cannot be loaded, importing this module fails.
"""
from __future__ import annotations

import array
import ctypes as C
import operator
import os
from typing import Optional

import torch

from . import build as _build

ROUND_NEAREST = 0
ROUND_STOCHASTIC = 1
FLAG_NO_MERGE = 1
FLAG_NO_SPLIT_K = 2
FLAG_RELU = 4
AMAX_HISTORY_WORDS = 1024
DTYPE_CODES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # hdqt_dtype_t
ACT_CODES = {"none": 0, "relu": 1, "silu": 2}                           # hdqt_act_t
REDUCE_CODES = {"none": 0, "mean": 1, "sum": 2}                         # HDQT_REDUCE_*
XENT_FWD, XENT_BWD, XENT_TRAIN = 0, 1, 2
NORM_CODES = {2.0: 2, float("inf"): 0}                                  # HDQT_NORM_*

STATUS_NAMES = ["OK", "INVALID_ARG", "UNSUPPORTED", "ALIGNMENT", "WORKSPACE", "NONFINITE", "TIMEOUT", "CUDA",
                "STATIC_SCRATCH"]

EXPORTED = [
    "hdqt_default_desc", "hdqt_padded_k", "hdqt_status_string", "hdqt_absmax_hadamard",
    "hdqt_quantize_hadamard", "hdqt_quantize_workspace_bytes", "hdqt_gemm_i8_tiled",
    "hdqt_gemm_i8_workspace_bytes", "hdqt_calibrate_acc_shift", "hdqt_gemm_fwd", "hdqt_gemm_dgrad",
    "hdqt_gemm_wgrad", "hdqt_workspace_bytes", "hdqt_workspace_layout", "hdqt_quantize_hadamard_static",
    "hdqt_selftest_bounded_wait", "hdqt_conv2d_fwd", "hdqt_conv2d_wgrad", "hdqt_selftest_mma_rate",
    "hdqt_grad_norm", "hdqt_clip_grad_norm", "hdqt_grad_norm_workspace_bytes", "hdqt_scale_tensors",
    "hdqt_group_norm_fwd", "hdqt_group_norm_bwd", "hdqt_group_norm_workspace_bytes",
    "hdqt_layer_norm_fwd", "hdqt_layer_norm_bwd", "hdqt_layer_norm_workspace_bytes", "hdqt_dropout_add",
    "hdqt_dropout_add_layer_norm_fwd", "hdqt_dropout_add_layer_norm_bwd",
    "hdqt_linear_xent_fwd", "hdqt_linear_xent_bwd", "hdqt_linear_xent_train", "hdqt_linear_xent_workspace_bytes",
]


class GemmDesc(C.Structure):
    """Mirror of hdqt_gemm_desc_t."""
    _fields_ = [
        ("in_bits", C.c_int32), ("acc_bits", C.c_int32), ("acc_tile", C.c_int32), ("acc_shift", C.c_int32),
        ("had_block", C.c_int32), ("clip_a", C.c_float), ("clip_b", C.c_float),
        ("round_a", C.c_int32), ("round_b", C.c_int32), ("seed", C.c_uint64),
        ("tag_a", C.c_uint32), ("tag_b", C.c_uint32), ("amax_a", C.c_void_p), ("amax_b", C.c_void_p),
        ("flags", C.c_uint32), ("bias", C.c_void_p),
        ("amax_hist_in_a", C.c_void_p), ("amax_hist_in_b", C.c_void_p),
        ("amax_hist_out_a", C.c_void_p), ("amax_hist_out_b", C.c_void_p),
        ("philox_offset", C.c_void_p),
    ]


class Conv2dGeom(C.Structure):
    """Mirror of hdqt_conv2d_geom_t."""
    _fields_ = [("batch", C.c_int64), ("height", C.c_int64), ("width", C.c_int64), ("channels", C.c_int64),
                ("kernel_h", C.c_int32), ("kernel_w", C.c_int32), ("stride", C.c_int32), ("padding", C.c_int32)]


class GroupNormDesc(C.Structure):
    """Mirror of hdqt_group_norm_desc_t."""
    _fields_ = [(n, C.c_int64) for n in ("batch", "pixels", "channels", "groups", "x_batch_stride", "x_pixel_stride",
                                         "y_batch_stride", "y_pixel_stride")] + \
               [("dtype", C.c_int32), ("param_dtype", C.c_int32), ("act", C.c_int32), ("eps", C.c_float)]


class LayerNormDesc(C.Structure):
    """Mirror of hdqt_layer_norm_desc_t."""
    _fields_ = [(n, C.c_int64) for n in ("rows", "channels", "x_row_stride", "r_row_stride", "y_row_stride")] + \
               [("dtype", C.c_int32), ("param_dtype", C.c_int32), ("act", C.c_int32), ("eps", C.c_float),
                ("p", C.c_double), ("seed", C.c_uint64), ("philox_offset", C.c_void_p), ("tag", C.c_uint32),
                ("reserved", C.c_uint32)]


class DropoutDesc(C.Structure):
    """Mirror of hdqt_dropout_desc_t."""
    _fields_ = [(n, C.c_int64) for n in ("rows", "cols", "x_row_stride", "r_row_stride", "y_row_stride")] + \
               [("p", C.c_double), ("seed", C.c_uint64), ("philox_offset", C.c_void_p), ("tag", C.c_uint32),
                ("dtype", C.c_int32)]


class XentDesc(C.Structure):
    """Mirror of hdqt_xent_desc_t."""
    _fields_ = [(n, C.c_int64) for n in ("tokens", "features", "classes", "ld_x", "ld_w", "ld_dx", "ld_dw",
                                         "ignore_index", "piece_bytes")] + \
               [(n, C.c_int32) for n in ("dtype", "w_is_cd", "reduction", "reserved")]


class WsLayout(C.Structure):
    """Mirror of hdqt_ws_layout_t."""
    _fields_ = [(n, C.c_size_t) for n in ("codes_a", "codes_b", "step_a", "step_b", "amax_a", "amax_b",
                                          "norms_a", "norms_b", "gemm_ws", "total")] + [("k_pad", C.c_int64)]


def _load() -> C.CDLL:
    path = _build.LIB_PATH
    if not os.path.exists(path) or _build.needs_rebuild():
        try:
            _build.build()
        except Exception as e:
            # No silent fallback: neither to a CPU path nor to a library older than the sources beside it.
            # A box without the CUDA toolkit may still load a library that was built elsewhere from these
            # very sources (the build stamps their digest next to it).
            if not (os.path.exists(path) and _build.stamp_matches_sources()):
                raise ImportError(f"HDQT CUDA library is missing or older than its sources and could not be "
                                  f"rebuilt: {e}") from e
    lib = C.CDLL(path)
    i32, i64, u32, u64, f32, vp, sz = C.c_int32, C.c_int64, C.c_uint32, C.c_uint64, C.c_float, C.c_void_p, C.c_size_t
    lib.hdqt_default_desc.argtypes = [C.POINTER(GemmDesc), C.c_int]
    lib.hdqt_default_desc.restype = None
    lib.hdqt_padded_k.argtypes = [i64, i32]
    lib.hdqt_padded_k.restype = i64
    lib.hdqt_status_string.argtypes = [C.c_int]
    lib.hdqt_status_string.restype = C.c_char_p
    lib.hdqt_absmax_hadamard.argtypes = [vp, i64, i64, i64, i64, i32, vp, vp, vp]
    lib.hdqt_quantize_hadamard.argtypes = [vp, i64, i64, i64, i64, i32, i32, f32, i32, u64, u32, vp, vp, vp, vp,
                                           vp, sz, vp, vp]
    lib.hdqt_quantize_hadamard_static.argtypes = [vp, i64, i64, i64, i64, i32, i32, f32, i32, u64, u32, vp, vp, vp,
                                                  vp, vp]
    lib.hdqt_quantize_hadamard_static.restype = C.c_int
    lib.hdqt_quantize_workspace_bytes.argtypes = [i64, i64, i32]
    lib.hdqt_quantize_workspace_bytes.restype = sz
    lib.hdqt_gemm_i8_tiled.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, i32, i32, i32, i32, vp, i64, vp, vp, i32,
                                       vp, vp, u32, vp, sz, vp, vp]
    lib.hdqt_gemm_i8_workspace_bytes.argtypes = [i64, i64, i64]
    lib.hdqt_gemm_i8_workspace_bytes.restype = sz
    lib.hdqt_calibrate_acc_shift.argtypes = [vp, vp, i64, i64, i64, i32, i32, vp, vp, sz, vp, vp]
    for name in ("hdqt_gemm_fwd", "hdqt_gemm_dgrad", "hdqt_gemm_wgrad"):
        getattr(lib, name).argtypes = [C.POINTER(GemmDesc), vp, vp, vp, i64, i64, i64, i32, vp, sz, vp, vp]
    lib.hdqt_selftest_mma_rate.argtypes = [i32, C.POINTER(C.c_int64), vp, vp]
    lib.hdqt_selftest_mma_rate.restype = C.c_int
    lib.hdqt_selftest_bounded_wait.argtypes = [vp, vp, vp]
    lib.hdqt_selftest_bounded_wait.restype = C.c_int
    for name in ("hdqt_conv2d_fwd", "hdqt_conv2d_wgrad"):
        getattr(lib, name).argtypes = [C.POINTER(GemmDesc), C.POINTER(Conv2dGeom), vp, vp, vp, i64, vp, sz, vp, vp]
        getattr(lib, name).restype = C.c_int
    lib.hdqt_grad_norm.argtypes = [vp, i64, i32, vp, vp, sz, vp]
    lib.hdqt_clip_grad_norm.argtypes = [vp, i64, i32, f32, vp, vp, sz, vp]
    lib.hdqt_grad_norm_workspace_bytes.argtypes = [i64]
    lib.hdqt_scale_tensors.argtypes = [vp, i64, vp, vp]
    lib.hdqt_scale_tensors.restype = C.c_int
    lib.hdqt_grad_norm_workspace_bytes.restype = sz
    lib.hdqt_group_norm_fwd.argtypes = [C.POINTER(GroupNormDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hdqt_group_norm_bwd.argtypes = [C.POINTER(GroupNormDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hdqt_group_norm_workspace_bytes.argtypes = [C.POINTER(GroupNormDesc), i32]
    lib.hdqt_group_norm_workspace_bytes.restype = sz
    lib.hdqt_layer_norm_fwd.argtypes = [C.POINTER(LayerNormDesc), vp, vp, vp, vp, vp, vp, vp]
    lib.hdqt_layer_norm_bwd.argtypes = [C.POINTER(LayerNormDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hdqt_layer_norm_workspace_bytes.argtypes = [C.POINTER(LayerNormDesc)]
    lib.hdqt_layer_norm_workspace_bytes.restype = sz
    lib.hdqt_dropout_add.argtypes = [C.POINTER(DropoutDesc), vp, vp, vp, vp]
    lib.hdqt_dropout_add_layer_norm_fwd.argtypes = [C.POINTER(LayerNormDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.hdqt_dropout_add_layer_norm_bwd.argtypes = [C.POINTER(LayerNormDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                    vp, sz, vp]
    for name in ("hdqt_layer_norm_fwd", "hdqt_layer_norm_bwd", "hdqt_dropout_add", "hdqt_dropout_add_layer_norm_fwd",
                 "hdqt_dropout_add_layer_norm_bwd"):
        getattr(lib, name).restype = C.c_int
    lib.hdqt_linear_xent_fwd.argtypes = [C.POINTER(XentDesc), vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.hdqt_linear_xent_bwd.argtypes = [C.POINTER(XentDesc), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.hdqt_linear_xent_train.argtypes = [C.POINTER(XentDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.hdqt_linear_xent_workspace_bytes.argtypes = [C.POINTER(XentDesc), i32]
    lib.hdqt_linear_xent_workspace_bytes.restype = sz
    for name in ("hdqt_linear_xent_fwd", "hdqt_linear_xent_bwd", "hdqt_linear_xent_train"):
        getattr(lib, name).restype = C.c_int
    for name in ("hdqt_grad_norm", "hdqt_clip_grad_norm", "hdqt_group_norm_fwd", "hdqt_group_norm_bwd"):
        getattr(lib, name).restype = C.c_int
    lib.hdqt_workspace_bytes.argtypes = [C.POINTER(GemmDesc), i64, i64, i64]
    lib.hdqt_workspace_bytes.restype = sz
    lib.hdqt_workspace_layout.argtypes = [C.POINTER(GemmDesc), i64, i64, i64, C.POINTER(WsLayout)]
    for name in ("hdqt_absmax_hadamard", "hdqt_quantize_hadamard", "hdqt_gemm_i8_tiled", "hdqt_calibrate_acc_shift",
                 "hdqt_gemm_fwd", "hdqt_gemm_dgrad", "hdqt_gemm_wgrad", "hdqt_workspace_layout"):
        getattr(lib, name).restype = C.c_int
    return lib


lib = _load()


class HdqtError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib.hdqt_status_string(status).decode()} (status {status})")


def _check(status: int, where: str) -> None:
    if status != 0:
        raise HdqtError(status, where)


# the raw handle of a device's current stream without a Stream object around it (0.2 us instead of 3 per call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_raw_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream() -> int:
    return _raw_stream(_raw_device())


def _call(name: str, t: torch.Tensor, *args) -> None:
    """The C entry `name` with `args` and a stream, on t's device: the library launches on the current device, which is made t's
    for the call where it is another one."""
    index = t.get_device()
    if index == _raw_device():
        status = getattr(lib, name)(*args, _raw_stream(index))
    elif index < 0:
        raise ValueError("expected CUDA tensors")
    else:
        with torch.cuda.device(index):
            status = getattr(lib, name)(*args, _raw_stream(index))
    _check(status, name)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _status(t: Optional[torch.Tensor], like: torch.Tensor) -> Optional[int]:
    if t is None:
        return None
    if t.device != like.device or t.dtype != torch.int32 or t.numel() < 1:
        raise ValueError("dev_status must be an int32 tensor on the operands' device (new_status)")
    return t.data_ptr()


def new_status(device) -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


def check_device_status(dev_status: torch.Tensor, where: str = "hdqt") -> None:
    """Synchronises and raises if a kernel recorded an error."""
    code = int(dev_status.item())
    if code != 0:
        raise HdqtError(code, where)


def default_desc(kind: str, **overrides) -> GemmDesc:
    d = GemmDesc()
    lib.hdqt_default_desc(C.byref(d), {"fwd": 0, "dgrad": 1, "wgrad": 2}[kind])
    for k, v in overrides.items():
        if k in ("amax_a", "amax_b", "bias", "amax_hist_in_a", "amax_hist_in_b", "amax_hist_out_a", "amax_hist_out_b",
                 "philox_offset"):
            v = _ptr(v)
        setattr(d, k, v)
    return d


def padded_k(K: int, had_block: int = 32) -> int:
    return int(lib.hdqt_padded_k(K, had_block))


def _view_2d(src: torch.Tensor):
    """(rows, K, ld_row, ld_k) of a 2-D fp32 CUDA tensor whose dim 1 is the contraction index."""
    if src.dim() != 2 or src.dtype != torch.float32 or not src.is_cuda:
        raise ValueError("expected a 2-D fp32 CUDA tensor")
    rows, K = src.shape
    ld_row, ld_k = src.stride()
    if K == 1 and ld_k != 1:
        ld_k = 1
    if rows == 1 and ld_row != 1 and ld_k != 1:
        ld_row = 1
    return rows, K, ld_row, ld_k


def absmax_hadamard(src: torch.Tensor, had_block: int = 32, dev_status: Optional[torch.Tensor] = None):
    rows, K, ld_row, ld_k = _view_2d(src)
    out = torch.empty(1, dtype=torch.float32, device=src.device)
    _call("hdqt_absmax_hadamard", src, src.data_ptr(), rows, K, ld_row, ld_k, had_block, out.data_ptr(),
          _ptr(dev_status))
    return out


def quantize_hadamard(src: torch.Tensor, had_block: int = 32, bits: int = 4, clip: float = 1.0,
                      mode: int = ROUND_NEAREST, seed: int = 0, tag: int = 0,
                      amax: Optional[torch.Tensor] = None, want_norms: bool = False,
                      dev_status: Optional[torch.Tensor] = None, out=None):
    """src[rows, K] (dim 1 = contraction; either dim may be the contiguous one).
    Returns (codes int8 [rows, K_pad], step fp32 [1], tile_norms int32 or None)."""
    rows, K, ld_row, ld_k = _view_2d(src)
    Kp = padded_k(K, had_block)
    if out is None:
        codes = torch.empty((rows, Kp), dtype=torch.int8, device=src.device)
        step = torch.empty(1, dtype=torch.float32, device=src.device)
        norms = torch.empty(((rows + 127) // 128, Kp // 32), dtype=torch.int32, device=src.device) if want_norms else None
        ws = torch.empty(lib.hdqt_quantize_workspace_bytes(rows, K, had_block), dtype=torch.uint8, device=src.device)
    else:
        codes, step, norms, ws = out
    _call("hdqt_quantize_hadamard", src, src.data_ptr(), rows, K, ld_row, ld_k, had_block, bits, clip, mode, seed,
          tag, _ptr(amax), codes.data_ptr(), step.data_ptr(), _ptr(norms), ws.data_ptr(), ws.numel(),
          _ptr(dev_status))
    return codes, step, norms


STATIC_SCRATCH_BYTES = 256 + 4096
STATIC_MAX_ROW_TILES = 2097152


def quantize_hadamard_static(src: torch.Tensor, codes: torch.Tensor, step: torch.Tensor,
                             norms: Optional[torch.Tensor] = None, had_block: int = 32, bits: int = 4,
                             clip: float = 1.0, mode: int = ROUND_NEAREST, seed: int = 0, tag: int = 0,
                             dev_status: Optional[torch.Tensor] = None):
    """Same result as quantize_hadamard (measured maximum), written into buffers the caller already
    owns, for callers that cannot allocate device memory at this point: the library's built-in
    scratch array replaces the workspace, so neither this wrapper nor the C call allocates anything.
    Operands are limited to rows * K_pad / 32 <= 2 097 152; calls on different streams must not
    overlap (they share the one array)."""
    rows, K, ld_row, ld_k = _view_2d(src)
    _call("hdqt_quantize_hadamard_static", src, src.data_ptr(), rows, K, ld_row, ld_k, had_block, bits, clip, mode,
          seed, tag, codes.data_ptr(), step.data_ptr(), _ptr(norms), _ptr(dev_status))
    return codes, step, norms


def gemm_i8_tiled(Aq: torch.Tensor, Bq: torch.Tensor, step_a: torch.Tensor, step_b: torch.Tensor,
                  acc_bits: int = 8, acc_tile: int = 32, acc_shift: int = 0, had_block: int = 32,
                  code_bits: int = 4, want_S: bool = False, want_tiles: bool = False, norms_a=None, norms_b=None, flags: int = 0,
                  dev_status: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """Out[M,N] from codes Aq[M,K_pad], Bq[N,K_pad]. Returns (out, S or None, tiles or None)."""
    M, Kp = Aq.shape
    N, Kp2 = Bq.shape
    if Kp != Kp2 or Aq.dtype != torch.int8 or Bq.dtype != torch.int8:
        raise ValueError("code matrices must be int8 with equal K_pad")
    if not (Aq.is_contiguous() and Bq.is_contiguous()):
        raise ValueError("code matrices must be contiguous")
    dev = Aq.device
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=dev)
    S = torch.empty((M, N), dtype=torch.int32, device=dev) if want_S else None
    tiles, elem = None, 0
    if want_tiles:
        s = acc_tile if acc_tile else Kp
        T = (Kp + s - 1) // s
        elem = 1 if acc_bits <= 8 else 2
        tiles = torch.empty((T, M, N), dtype=torch.int8 if elem == 1 else torch.int16, device=dev)
    ws = torch.empty(max(256, lib.hdqt_gemm_i8_workspace_bytes(M, N, Kp)), dtype=torch.uint8, device=dev)
    _call("hdqt_gemm_i8_tiled", Aq, Aq.data_ptr(), Bq.data_ptr(), step_a.data_ptr(), step_b.data_ptr(), M, N, Kp,
          code_bits, acc_bits, acc_tile, acc_shift, had_block, out.data_ptr(), out.stride(0), _ptr(S), _ptr(tiles),
          elem, _ptr(norms_a), _ptr(norms_b), flags, ws.data_ptr(), ws.numel(), _ptr(dev_status))
    return out, S, tiles


def calibrate_acc_shift(Aq: torch.Tensor, Bq: torch.Tensor, acc_bits: int = 8, acc_tile: int = 32) -> torch.Tensor:
    M, Kp = Aq.shape
    N = Bq.shape[0]
    out = torch.empty(1, dtype=torch.int32, device=Aq.device)
    _call("hdqt_calibrate_acc_shift", Aq, Aq.data_ptr(), Bq.data_ptr(), M, N, Kp, acc_bits, acc_tile, out.data_ptr(),
          None, 0, None)
    return out


# ---- the three training GEMMs ---------------------------------------------------------------------

def workspace_layout(desc: GemmDesc, M: int, N: int, K: int) -> WsLayout:
    L = WsLayout()
    _check(lib.hdqt_workspace_layout(C.byref(desc), M, N, K, C.byref(L)), "hdqt_workspace_layout")
    return L


def workspace_bytes(desc: GemmDesc, M: int, N: int, K: int) -> int:
    return int(lib.hdqt_workspace_bytes(C.byref(desc), M, N, K))


class Workspace:
    """A device buffer plus the layout the library carves it into (to read intermediates back)."""

    def __init__(self, desc: GemmDesc, M: int, N: int, K: int, device):
        self.layout = workspace_layout(desc, M, N, K)
        self.M, self.N = M, N
        self.buf = torch.empty(self.layout.total, dtype=torch.uint8, device=device)

    def codes_a(self):
        L = self.layout
        return self.buf[L.codes_a:L.codes_a + self.M * L.k_pad].view(torch.int8).view(self.M, L.k_pad)

    def codes_b(self):
        L = self.layout
        return self.buf[L.codes_b:L.codes_b + self.N * L.k_pad].view(torch.int8).view(self.N, L.k_pad)

    def scalar(self, name: str) -> torch.Tensor:
        off = getattr(self.layout, name)
        return self.buf[off:off + 4].view(torch.float32)


def _w_dims(W: torch.Tensor, w_is_cd: bool):
    return (W.shape[1], W.shape[0]) if w_is_cd else (W.shape[0], W.shape[1])


def _run(fn_name, desc, a, b, out, Nb, D, C_, w_is_cd, M, N, K, workspace, dev_status):
    if workspace is None:
        workspace = Workspace(desc, M, N, K, a.device)
    _call(fn_name, a, C.byref(desc), a.data_ptr(), b.data_ptr(), out.data_ptr(), Nb, D, C_, 1 if w_is_cd else 0,
          workspace.buf.data_ptr(), workspace.buf.numel(), _ptr(dev_status))
    return out, workspace


def _req(t: torch.Tensor, name: str):
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 CUDA tensor")


def gemm_fwd(X, W, desc: Optional[GemmDesc] = None, w_is_cd: bool = False, workspace=None, dev_status=None,
             out=None):
    """Y[Nb,C] = X[Nb,D] W. W is [D,C], or [C,D] when w_is_cd. Returns (Y, workspace)."""
    _req(X, "X"); _req(W, "W")
    desc = desc or default_desc("fwd")
    Nb, D = X.shape
    Dw, Cw = _w_dims(W, w_is_cd)
    if Dw != D:
        raise ValueError("shape mismatch")
    if out is None:
        out = torch.empty((Nb, Cw), dtype=torch.float32, device=X.device)
    return _run("hdqt_gemm_fwd", desc, X, W, out, Nb, D, Cw, w_is_cd, Nb, Cw, D, workspace, dev_status)


def gemm_dgrad(G, W, desc: Optional[GemmDesc] = None, w_is_cd: bool = False, workspace=None, dev_status=None,
               out=None):
    """dX[Nb,D] = G[Nb,C] W^T. Returns (dX, workspace)."""
    _req(G, "G"); _req(W, "W")
    desc = desc or default_desc("dgrad")
    Nb, Cg = G.shape
    Dw, Cw = _w_dims(W, w_is_cd)
    if Cw != Cg:
        raise ValueError("shape mismatch")
    if out is None:
        out = torch.empty((Nb, Dw), dtype=torch.float32, device=G.device)
    return _run("hdqt_gemm_dgrad", desc, G, W, out, Nb, Dw, Cg, w_is_cd, Nb, Dw, Cg, workspace, dev_status)


def gemm_wgrad(X, G, desc: Optional[GemmDesc] = None, w_is_cd: bool = False, workspace=None, dev_status=None,
               out=None):
    """dW = X^T G in W's layout ([D,C], or [C,D] when w_is_cd). Returns (dW, workspace)."""
    _req(X, "X"); _req(G, "G")
    desc = desc or default_desc("wgrad")
    Nb, D = X.shape
    Nb2, Cg = G.shape
    if Nb != Nb2:
        raise ValueError("shape mismatch")
    M, N = (Cg, D) if w_is_cd else (D, Cg)
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    return _run("hdqt_gemm_wgrad", desc, X, G, out, Nb, D, Cg, w_is_cd, M, N, Nb, workspace, dev_status)


# ---- convolution without a materialised patch matrix ------------------------------------------------

def conv2d_out_size(H: int, W: int, kernel, stride: int, padding: int):
    """Output height and width; `kernel` is an int (square) or a (kh, kw) pair."""
    kh, kw = (kernel, kernel) if isinstance(kernel, int) else kernel
    return (H + 2 * padding - kh) // stride + 1, (W + 2 * padding - kw) // stride + 1


def conv2d_fwd(X, W, stride: int = 1, padding: int = 0, desc: Optional[GemmDesc] = None, workspace=None,
               dev_status=None, out=None):
    """Y[B,Ho,Wo,Cout] from X[B,H,W,Cin] (NHWC, Cin % 32 == 0) and W[Cout,kh,kw,Cin]. Returns (Y, workspace)."""
    _req(X, "X"); _req(W, "W")
    desc = desc or default_desc("fwd")
    B, H, Wd, Cin = X.shape
    Cout, kh, kw, Cin2 = W.shape
    if Cin2 != Cin:
        raise ValueError("shape mismatch")
    Ho, Wo = conv2d_out_size(H, Wd, (kh, kw), stride, padding)
    g = Conv2dGeom(B, H, Wd, Cin, kh, kw, stride, padding)
    M, N, K = B * Ho * Wo, Cout, kh * kw * Cin
    if workspace is None:
        workspace = Workspace(desc, M, N, K, X.device)
    if out is None:
        out = torch.empty((B, Ho, Wo, Cout), dtype=torch.float32, device=X.device)
    _call("hdqt_conv2d_fwd", X, C.byref(desc), C.byref(g), X.data_ptr(), W.data_ptr(), out.data_ptr(), Cout,
          workspace.buf.data_ptr(), workspace.buf.numel(), _ptr(dev_status))
    return out, workspace


def conv2d_dgrad(G, W, padding: int = 0, desc: Optional[GemmDesc] = None, workspace=None, dev_status=None, out=None):
    """dX[B,H,W,Cin] of a stride-1 convolution from G[B,Ho,Wo,Cout] (NHWC, Cout % 32 == 0) and W[Cout,kh,kw,Cin]:
    the input gradient is itself a convolution, of G with the kernel rotated by 180 degrees and padding
    k-1-padding, so it runs through hdqt_conv2d_fwd with the dgrad roles (stochastic rounding on G, nearest on
    W): contraction over (kh, kw, cout), no patch-matrix gradient and no scatter-add.  Returns (dX, workspace)."""
    _req(G, "G"); _req(W, "W")
    desc = desc or default_desc("dgrad")
    Cout, kh, kw, Cin = W.shape
    if G.shape[3] != Cout or kh - 1 - padding != kw - 1 - padding or kh - 1 - padding < 0:
        raise ValueError("shape mismatch")
    w_rot = W.flip(1, 2).permute(3, 1, 2, 0).contiguous()          # [Cin, kh, kw, Cout]
    return conv2d_fwd(G, w_rot, 1, kh - 1 - padding, desc=desc, workspace=workspace, dev_status=dev_status, out=out)


def conv2d_wgrad(X, G, kernel, stride: int = 1, padding: int = 0, desc: Optional[GemmDesc] = None,
                 workspace=None, dev_status=None, out=None):
    """dW[Cout,kh,kw,Cin] from X[B,H,W,Cin] and G[B,Ho,Wo,Cout] (both NHWC); `kernel` is an int or (kh, kw).
    Returns (dW, workspace)."""
    _req(X, "X"); _req(G, "G")
    desc = desc or default_desc("wgrad")
    B, H, Wd, Cin = X.shape
    Cout = G.shape[3]
    kh, kw = (kernel, kernel) if isinstance(kernel, int) else kernel
    Ho, Wo = conv2d_out_size(H, Wd, (kh, kw), stride, padding)
    if tuple(G.shape[:3]) != (B, Ho, Wo):
        raise ValueError("shape mismatch")
    g = Conv2dGeom(B, H, Wd, Cin, kh, kw, stride, padding)
    M, N, K = Cout, kh * kw * Cin, B * Ho * Wo
    if workspace is None:
        workspace = Workspace(desc, M, N, K, X.device)
    if out is None:
        out = torch.empty((Cout, kh, kw, Cin), dtype=torch.float32, device=X.device)
    _call("hdqt_conv2d_wgrad", X, C.byref(desc), C.byref(g), X.data_ptr(), G.data_ptr(), out.data_ptr(), Cout,
          workspace.buf.data_ptr(), workspace.buf.numel(), _ptr(dev_status))
    return out, workspace


def mma_rate_tops(iters: int = 20000, repeats: int = 3, dev_status=None) -> float:
    """Integer tensor rate (TOP/s) of back-to-back M128 N256 K32 kind::i8 MMAs on all SMs (no loads, no epilogue),
    best of `repeats` timed launches: the ceiling of the tiled GEMM at the current clocks."""
    ops = C.c_int64(0)
    best = 0.0
    for _ in range(repeats + 1):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        _check(lib.hdqt_selftest_mma_rate(iters, C.byref(ops), _ptr(dev_status), _stream()), "hdqt_selftest_mma_rate")
        e1.record()
        torch.cuda.synchronize()
        best = max(best, ops.value / (e0.elapsed_time(e1) * 1e-3) / 1e12)
    return best


# ---- the rest of a training step: gradient clipping, group norm --------------------------------------

_dtype_of = operator.attrgetter("dtype")


def _tensor_table(tensors, out):
    """hdqt_tensor_t[len(tensors)] as a flat int64 array (source, destination, elements, type), and the device.  One pass
    per property: a model has hundreds of tensors, and this is most of the call's host time."""
    n = len(tensors)
    T = torch.Tensor
    codes = list(map(DTYPE_CODES.get, map(_dtype_of, tensors)))
    sizes = list(map(T.numel, tensors))
    at = list(map(T.data_ptr, tensors))
    devices = set(map(T.get_device, tensors))
    if None in codes or -1 in devices or not all(map(T.is_contiguous, tensors)):
        raise ValueError("expected dense fp32, bf16 or fp16 CUDA tensors")
    to = at
    if out is not None:
        if len(out) != n or list(map(T.numel, out)) != sizes or list(map(DTYPE_CODES.get, map(_dtype_of, out))) != codes \
                or not all(map(T.is_contiguous, out)):
            raise ValueError("out must hold a dense tensor of the type and size of each input")
        devices.update(map(T.get_device, out))
        to = list(map(T.data_ptr, out))
    if len(devices) > 1:
        raise ValueError("the tensors must be on one device")
    table = array.array("q", bytes(32 * n))
    table[0::4] = array.array("q", at)
    table[1::4] = array.array("q", to)
    table[2::4] = array.array("q", sizes)
    table[3::4] = array.array("q", codes)
    return table, torch.device("cuda", devices.pop()) if devices else None


def _norm_code(norm_type) -> int:
    code = NORM_CODES.get(float(norm_type))
    if code is None:
        raise ValueError("norm_type must be 2 or inf")
    return code


def grad_norm(tensors, norm_type: float = 2.0, device=None) -> torch.Tensor:
    """Norm over all elements of a list of dense fp32 / bf16 / fp16 tensors (types may be mixed), as an fp32 scalar
    tensor: 2 = Euclidean, inf = largest magnitude.  `device` is needed for an empty list only."""
    tensors = list(tensors)
    code = _norm_code(norm_type)
    table, dev = _tensor_table(tensors, None)
    dev = dev if dev is not None else torch.device(device or "cuda")
    norm = torch.empty((), dtype=torch.float32, device=dev)
    nbytes = lib.hdqt_grad_norm_workspace_bytes(len(tensors))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _call("hdqt_grad_norm", norm, table.buffer_info()[0], len(tensors), code, norm.data_ptr(), ws.data_ptr(), nbytes)
    return norm


def clip_grad_norm(tensors, max_norm: float, norm_type: float = 2.0, out=None, device=None) -> torch.Tensor:
    """Scales the tensors by min(1, max_norm / (norm + 1e-6)), in place or into the tensors of `out`, and returns the
    norm they had (see grad_norm).  A tensor that is written may not overlap another one of the call.  Nothing synchronises
    the host; the call can be recorded into a CUDA graph."""
    tensors = list(tensors)
    code = _norm_code(norm_type)
    table, dev = _tensor_table(tensors, None if out is None else list(out))
    dev = dev if dev is not None else torch.device(device or "cuda")
    norm = torch.empty((), dtype=torch.float32, device=dev)
    nbytes = lib.hdqt_grad_norm_workspace_bytes(len(tensors))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _call("hdqt_clip_grad_norm", norm, table.buffer_info()[0], len(tensors), code, max_norm, norm.data_ptr(),
          ws.data_ptr(), nbytes)
    return norm


def scale_tensors(tensors, factor: torch.Tensor, out=None) -> None:
    """Multiplies dense tensors by an fp32 scalar tensor, in place or into the tensors of `out`; a factor of 1 in place costs
    one launch and no memory traffic."""
    tensors = list(tensors)
    table, dev = _tensor_table(tensors, None if out is None else list(out))
    if factor.dtype != torch.float32 or factor.numel() != 1 or (dev is not None and factor.device != dev):
        raise ValueError("factor must be an fp32 scalar on the tensors' device")
    _call("hdqt_scale_tensors", factor, table.buffer_info()[0], len(tensors), factor.data_ptr())


def _pixel_strides(t: torch.Tensor, name: str):
    """(batch stride, pixel stride) of a [batch, ..., channels] tensor whose inner dimensions step evenly."""
    shape, st = t.shape, t.stride()
    if len(shape) < 2:
        raise ValueError(f"{name} must be [batch, ..., channels]")
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must have its channels contiguous")
    if 0 in shape[1:-1]:                                       # no pixels: whatever the strides, nothing lies anywhere
        return 0, shape[-1]
    pixel, step = None, 0
    for size, stride in zip(shape[-2:0:-1], st[-2:0:-1]):      # pixel dimensions, innermost first
        if size == 1:
            continue
        if pixel is None:
            pixel = stride
        elif stride != step:
            raise ValueError(f"the pixels of {name} must be evenly spaced")
        step = stride * size
    if pixel is None:
        pixel = shape[-1]
        step = pixel
    batch = st[0] if shape[0] > 1 else step
    return batch, pixel


def _group_norm_desc(x, gamma, beta, groups: int, eps: float, act: str):
    """Checks, descriptor and workspace sizes of a call."""
    code = DTYPE_CODES.get(x.dtype)
    if code is None or not x.is_cuda:
        raise ValueError("expected an fp32, bf16 or fp16 CUDA tensor")
    if act not in ACT_CODES:
        raise ValueError(f"act must be one of {sorted(ACT_CODES)}")
    channels = x.shape[-1]
    pdt = x.dtype
    for t in (gamma, beta):
        if t is None:
            continue
        if t.shape != (channels,) or not t.is_contiguous():
            raise ValueError("gamma and beta must be dense [channels] tensors")
        pdt = t.dtype
    if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
        raise ValueError("gamma and beta must have one type")
    if pdt not in (torch.float32, x.dtype):
        raise ValueError("gamma and beta must be fp32 or of x's type")
    pixels = 1
    for n in x.shape[1:-1]:
        pixels *= n
    d = GroupNormDesc(x.shape[0], pixels, channels, groups, 0, 0, pixels * channels, channels, code, DTYPE_CODES[pdt],
                      ACT_CODES[act], eps)
    d.x_batch_stride, d.x_pixel_stride = _pixel_strides(x, "x")
    sizes = [max(256, lib.hdqt_group_norm_workspace_bytes(C.byref(d), i)) for i in (0, 1)]
    return d, sizes


_GROUP_NORM_PLANS = {}     # descriptor and workspace sizes by shapes, strides and types


def _group_norm_plan(x, gamma, beta, groups, eps, act):
    key = (x.shape, x.stride(), x.dtype, x.is_cuda, groups, eps, act,
           None if gamma is None else (gamma.shape, gamma.dtype, gamma.is_contiguous()),
           None if beta is None else (beta.shape, beta.dtype, beta.is_contiguous()))
    plan = _GROUP_NORM_PLANS.get(key)
    if plan is None:
        if len(_GROUP_NORM_PLANS) >= 1024:
            _GROUP_NORM_PLANS.clear()
        plan = _GROUP_NORM_PLANS[key] = _group_norm_desc(x, gamma, beta, groups, eps, act)
    dev = x.device
    if (gamma is not None and gamma.device != dev) or (beta is not None and beta.device != dev):
        raise ValueError("gamma and beta must be on x's device")
    return plan


def group_norm_fwd(x, gamma, beta, groups: int, eps: float = 1e-5, act: str = "none"):
    """act(group norm) of x[batch, ..., channels] (channels last, evenly spaced pixels: a channel slice is fine).
    gamma, beta: [channels], fp32 or x's type, or None.  act: "none", "relu" or "silu".
    Returns (y dense, mean fp32 [batch, groups], rstd fp32 [batch, groups])."""
    d, (nbytes, _) = _group_norm_plan(x, gamma, beta, groups, eps, act)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    stats = x.new_empty((2, d.batch, max(groups, 0)), dtype=torch.float32)
    mean, rstd = stats.unbind(0)
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    _call("hdqt_group_norm_fwd", x, C.byref(d), x.data_ptr(), _ptr(gamma), _ptr(beta), y.data_ptr(), mean.data_ptr(),
          rstd.data_ptr(), ws.data_ptr(), nbytes)
    return y, mean, rstd


def group_norm_bwd(dy, x, gamma, beta, mean, rstd, groups: int, act: str = "none", want_dx: bool = True,
                   want_params: bool = True):
    """Gradients of group_norm_fwd: (dx dense or None, dgamma or None, dbeta or None)."""
    d, (_, nbytes) = _group_norm_plan(x, gamma, beta, groups, 0.0, act)
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.device != x.device:
        raise ValueError("dy must have x's shape, type and device")
    if mean.shape != (d.batch, groups) or mean.shape != rstd.shape or mean.dtype != torch.float32 \
            or rstd.dtype != torch.float32 or not (mean.is_contiguous() and rstd.is_contiguous()) \
            or mean.device != x.device or rstd.device != x.device:
        raise ValueError("mean and rstd must be the dense fp32 [batch, groups] tensors of the forward call")
    if not dy.is_contiguous():
        dy = dy.contiguous()
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want_dx else None
    dgamma = torch.empty_like(gamma) if want_params and gamma is not None else None
    dbeta = torch.empty_like(beta) if want_params and beta is not None else None
    ws = x.new_empty(nbytes, dtype=torch.uint8)
    _call("hdqt_group_norm_bwd", x, C.byref(d), dy.data_ptr(), x.data_ptr(), _ptr(gamma), _ptr(beta), mean.data_ptr(),
          rstd.data_ptr(), _ptr(dx), _ptr(dgamma), _ptr(dbeta), ws.data_ptr(), nbytes)
    return dx, dgamma, dbeta


# ---- layer norm, dropout, and both on the residual stream ---------------------------------------------

def _row_stride(t: torch.Tensor, name: str):
    """Elements between the rows of a [..., channels] tensor whose outer dimensions step evenly (the width itself for one row)."""
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    if t.is_contiguous():
        return shape[-1]
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must have its last dimension contiguous")
    row, step = None, 0
    for size, stride in zip(shape[-2::-1], st[-2::-1]):
        if size == 0:
            return shape[-1]
        if size == 1:
            continue
        if row is None:
            row = stride
            if row < shape[-1]:
                raise ValueError(f"the rows of {name} must not overlap")
        elif stride != step:
            raise ValueError(f"the rows of {name} must be evenly spaced")
        step = stride * size
    return shape[-1] if row is None else row


def _row_count(shape) -> int:
    rows = 1
    for n in shape[:-1]:
        rows *= n
    return rows


def _row_operand(t, x, name):
    """Raises unless t has x's shape, type and device."""
    if t.shape != x.shape or t.dtype is not x.dtype or t.get_device() != x.get_device():
        raise ValueError(f"{name} must have x's shape, type and device")


def _dropout_args(p, seed, tag, philox_offset, index):
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError("p must be a probability")
    if not 0 <= seed < 1 << 64 or not 0 <= tag < 1 << 32:
        raise ValueError("seed must fit 64 bits and tag 32 bits, both unsigned")
    if philox_offset is None:
        return p, None
    if philox_offset.dtype is not torch.int32 or philox_offset.numel() < 1 or philox_offset.get_device() != index:
        raise ValueError("philox_offset must be an int32 tensor on x's device")
    return p, philox_offset.data_ptr()


def _layer_norm_desc(x, gamma, beta, eps, act):
    code = DTYPE_CODES.get(x.dtype)
    if code is None or not x.is_cuda:
        raise ValueError("expected an fp32, bf16 or fp16 CUDA tensor")
    if act not in ACT_CODES:
        raise ValueError(f"act must be one of {sorted(ACT_CODES)}")
    stride = _row_stride(x, "x")
    channels = x.shape[-1]
    if channels == 0:
        raise ValueError("x must have at least one channel")
    pdt = x.dtype
    for t in (gamma, beta):
        if t is None:
            continue
        if t.shape != (channels,) or not t.is_contiguous():
            raise ValueError("gamma and beta must be dense [channels] tensors")
        pdt = t.dtype
    if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
        raise ValueError("gamma and beta must have one type")
    if pdt not in (torch.float32, x.dtype):
        raise ValueError("gamma and beta must be fp32 or of x's type")
    rows = _row_count(x.shape)
    d = LayerNormDesc(rows, channels, stride, channels, channels, code, DTYPE_CODES[pdt], ACT_CODES[act], eps, 0.0, 0, None, 0, 0)
    return d, lib.hdqt_layer_norm_workspace_bytes(C.byref(d)), tuple(x.shape[:-1])


_LAYER_NORM_PLANS = {}     # descriptor, workspace size and shape of the statistics by shapes, strides and types


def _layer_norm_plan(x, gamma, beta, eps, act):
    key = (x.shape, x.stride(), x.dtype, eps, act, None if gamma is None else (gamma.shape, gamma.stride(), gamma.dtype),
           None if beta is None else (beta.shape, beta.stride(), beta.dtype))
    plan = _LAYER_NORM_PLANS.get(key)
    if plan is None:
        plan = _layer_norm_desc(x, gamma, beta, eps, act)
        if len(_LAYER_NORM_PLANS) >= 1024:
            _LAYER_NORM_PLANS.clear()
        _LAYER_NORM_PLANS[key] = plan
    index = x.get_device()
    if index < 0:
        raise ValueError("expected CUDA tensors")
    if (gamma is not None and gamma.get_device() != index) or (beta is not None and beta.get_device() != index):
        raise ValueError("gamma and beta must be on x's device")
    return plan


def _check_stats(mean, rstd, shape, index):
    for t in (mean, rstd):
        if t.shape != shape or t.dtype is not torch.float32 or not t.is_contiguous() or t.get_device() != index:
            raise ValueError("mean and rstd must be the dense fp32 tensors of the forward call")


def _new_stats(shape, device):
    if not shape:      # one row
        return torch.empty((), dtype=torch.float32, device=device), torch.empty((), dtype=torch.float32, device=device)
    # (sizes as single arguments: a tuple takes torch another microsecond)
    return torch.empty(*shape, dtype=torch.float32, device=device), torch.empty(*shape, dtype=torch.float32, device=device)


def layer_norm_fwd(x, gamma, beta, eps: float = 1e-5, act: str = "none"):
    """act(layer norm) over the last dimension of x[..., channels] (evenly spaced rows: a slice of the channels is fine).
    gamma, beta: [channels], fp32 or x's type, or None.  act: "none", "relu" or "silu".
    Returns (y dense, mean fp32 [...], rstd fp32 [...])."""
    d, _, shape = _layer_norm_plan(x, gamma, beta, eps, act)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    mean, rstd = _new_stats(shape, x.device)
    _call("hdqt_layer_norm_fwd", x, C.byref(d), x.data_ptr(), _ptr(gamma), _ptr(beta), y.data_ptr(), mean.data_ptr(),
          rstd.data_ptr())
    return y, mean, rstd


def layer_norm_bwd(dy, x, gamma, beta, mean, rstd, act: str = "none", want_dx: bool = True, want_params: bool = True):
    """Gradients of layer_norm_fwd: (dx dense or None, dgamma or None, dbeta or None)."""
    d, nbytes, shape = _layer_norm_plan(x, gamma, beta, 0.0, act)
    _row_operand(dy, x, "dy")
    _check_stats(mean, rstd, shape, x.get_device())
    if not dy.is_contiguous():
        dy = dy.contiguous()
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want_dx else None
    dgamma = torch.empty_like(gamma) if want_params and gamma is not None else None
    dbeta = torch.empty_like(beta) if want_params and beta is not None else None
    ws = x.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _call("hdqt_layer_norm_bwd", x, C.byref(d), dy.data_ptr(), x.data_ptr(), _ptr(gamma), _ptr(beta), mean.data_ptr(),
          rstd.data_ptr(), _ptr(dx), _ptr(dgamma), _ptr(dbeta), _ptr(ws), nbytes)
    return dx, dgamma, dbeta


def dropout(x, p: float, seed: int, tag: int = 0, residual=None, philox_offset=None):
    """residual + dropout(x) (residual None: dropout alone) of x[..., cols], evenly spaced rows, as a dense tensor.  The random
    numbers are those of (seed, tag, the int32 device word philox_offset or 0) and an element's position in the dense tensor, so
    that the gradient of x is dropout(dy, p, seed, tag, philox_offset=...); no mask is stored.  Kept elements are divided by the
    probability 1 - rint(65536 p) / 65536 that is used."""
    code = DTYPE_CODES.get(x.dtype)
    if code is None or not x.is_cuda:
        raise ValueError("expected an fp32, bf16 or fp16 CUDA tensor")
    p, offset = _dropout_args(p, seed, tag, philox_offset, x.get_device())
    shape = x.shape
    if residual is not None:
        _row_operand(residual, x, "residual")
    if x.is_contiguous() and (residual is None or residual.is_contiguous()):
        n = x.numel()
        d = DropoutDesc(1, n, n, n, n, p, seed, offset, tag, code)
    else:
        cols = shape[-1] if shape else 1
        d = DropoutDesc(_row_count(shape), cols, _row_stride(x, "x"),
                        cols if residual is None else _row_stride(residual, "residual"), cols, p, seed, offset, tag, code)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    _call("hdqt_dropout_add", x, C.byref(d), x.data_ptr(), _ptr(residual), y.data_ptr())
    return y


def dropout_add_layer_norm_fwd(x, residual, gamma, beta, p: float, seed: int, tag: int = 0, eps: float = 1e-5,
                               act: str = "none", philox_offset=None):
    """h = residual + dropout(x) (residual may be None) and y = act(layer norm(h)) in one pass over the rows; arguments as in dropout
    and layer_norm_fwd.  Returns (y, h, mean, rstd), y and h dense."""
    d, _, shape = _layer_norm_plan(x, gamma, beta, eps, act)
    p, offset = _dropout_args(p, seed, tag, philox_offset, x.get_device())
    d = LayerNormDesc.from_buffer_copy(d)      # (a call of its own: plans are shared)
    d.p, d.seed, d.tag, d.philox_offset = p, seed, tag, offset
    if residual is not None:
        _row_operand(residual, x, "residual")
        d.r_row_stride = _row_stride(residual, "residual")
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    h = torch.empty_like(x, memory_format=torch.contiguous_format)
    mean, rstd = _new_stats(shape, x.device)
    _call("hdqt_dropout_add_layer_norm_fwd", x, C.byref(d), x.data_ptr(), _ptr(residual), _ptr(gamma), _ptr(beta), h.data_ptr(),
          y.data_ptr(), mean.data_ptr(), rstd.data_ptr())
    return y, h, mean, rstd


def dropout_add_layer_norm_bwd(dy, dh, h, gamma, beta, mean, rstd, p: float, seed: int, tag: int = 0, act: str = "none",
                               philox_offset=None, want_dx: bool = True, want_residual: bool = True,
                               want_params: bool = True):
    """Gradients of dropout_add_layer_norm_fwd from the h it returned (dense); dh: the gradient that arrives for h itself, or None.
    Returns (dx, dresidual, dgamma, dbeta), None where not wanted.  p, seed, tag, philox_offset as in the forward call (the device
    word must still hold the value it had then)."""
    d, nbytes, shape = _layer_norm_plan(h, gamma, beta, 0.0, act)
    p, offset = _dropout_args(p, seed, tag, philox_offset, h.get_device())
    if not h.is_contiguous():
        raise ValueError("h must be the dense tensor of the forward call")
    _row_operand(dy, h, "dy")
    _check_stats(mean, rstd, shape, h.get_device())
    if not dy.is_contiguous():
        dy = dy.contiguous()
    if dh is not None:
        _row_operand(dh, h, "dh")
        if not dh.is_contiguous():
            dh = dh.contiguous()
    d = LayerNormDesc.from_buffer_copy(d)
    d.p, d.seed, d.tag, d.philox_offset = p, seed, tag, offset
    dx = torch.empty_like(h) if want_dx else None
    dresidual = torch.empty_like(h) if want_residual else None
    dgamma = torch.empty_like(gamma) if want_params and gamma is not None else None
    dbeta = torch.empty_like(beta) if want_params and beta is not None else None
    ws = h.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _call("hdqt_dropout_add_layer_norm_bwd", h, C.byref(d), dy.data_ptr(), _ptr(dh), h.data_ptr(), _ptr(gamma), _ptr(beta),
          mean.data_ptr(), rstd.data_ptr(), _ptr(dx), _ptr(dresidual), _ptr(dgamma), _ptr(dbeta), _ptr(ws), nbytes)
    return dx, dresidual, dgamma, dbeta


# ---- linear layer + softmax cross entropy over a large vocabulary ------------------------------------

def _rows(t, name: str, shape=None):
    """A 2-D bf16 / fp32 CUDA tensor with contiguous rows that the library can read in place (bf16: rows from 16-byte
    boundaries on; a tensor that starts elsewhere is copied)."""
    if t.dim() != 2 or t.dtype not in (torch.float32, torch.bfloat16) or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-D fp32 or bf16 CUDA tensor")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape}")
    if (t.stride(1) != 1 and t.shape[1] > 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"the rows of {name} must be contiguous")
    if t.dtype == torch.bfloat16 and t.data_ptr() % 16:
        t = t.clone(memory_format=torch.contiguous_format)
    return t


def _ld(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


_XENT_PLANS = {}     # descriptor and workspace size by sizes, strides, types and options


def _xent_call(X, W, labels, ignore_index, reduction, w_is_cd, piece_bytes, kind):
    X, W = _rows(X, "X"), _rows(W, "W")
    key = (X.shape, X.stride(), X.dtype, W.shape, W.stride(), W.dtype, ignore_index, reduction, w_is_cd, piece_bytes, kind)
    plan = _XENT_PLANS.get(key)
    if plan is None:
        if reduction not in REDUCE_CODES:
            raise ValueError(f"reduction must be one of {sorted(REDUCE_CODES)}")
        T, D = X.shape
        V = W.shape[0] if w_is_cd else W.shape[1]
        if W.shape[1 if w_is_cd else 0] != D or W.dtype != X.dtype:
            raise ValueError("X [tokens, features] and W must agree in features and type")
        d = XentDesc(T, D, V, max(_ld(X), D), max(_ld(W), W.shape[1]), D, W.shape[1], ignore_index, piece_bytes,
                     DTYPE_CODES[X.dtype], int(w_is_cd), REDUCE_CODES[reduction], 0)
        if len(_XENT_PLANS) >= 1024:
            _XENT_PLANS.clear()
        plan = _XENT_PLANS[key] = (d, max(256, lib.hdqt_linear_xent_workspace_bytes(C.byref(d), kind)))
    if W.device != X.device or labels.device != X.device:
        raise ValueError("X, W and labels must be on one device")
    if labels.dim() != 1 or labels.shape[0] != X.shape[0] or labels.dtype != torch.int64:
        raise ValueError("labels must be an int64 [tokens] tensor")
    if not labels.is_contiguous():
        labels = labels.contiguous()
    d, nbytes = plan
    return X, W, labels, d, X.new_empty(nbytes, dtype=torch.uint8), nbytes


def _loss_weight(g, reduction, T, device):
    shape = (T,) if reduction == "none" else ()
    if g is None:
        if reduction == "none":
            raise ValueError("reduction 'none' needs the weight of each token's loss (g)")
        return None
    if tuple(g.shape) != shape or g.dtype != torch.float32 or g.device != device:
        raise ValueError(f"g must be an fp32 tensor of shape {shape} on X's device")
    return g.contiguous()


def linear_xent_fwd(X, W, labels, ignore_index: int = -100, reduction: str = "mean", w_is_cd: bool = False,
                    dev_status=None):
    """Softmax cross entropy of X[tokens, features] times W ([features, classes], or [classes, features] with w_is_cd)
    against int64 labels; the logits are not stored but for a few tokens or output blocks.  bf16 or fp32.  Returns (loss:
    scalar, or [tokens] with reduction "none"; lse fp32 [tokens])."""
    X, W, labels, d, ws, nbytes = _xent_call(X, W, labels, ignore_index, reduction, w_is_cd, 0, XENT_FWD)
    lse = X.new_empty(d.tokens, dtype=torch.float32)
    loss = X.new_empty((d.tokens,) if reduction == "none" else (), dtype=torch.float32)
    _call("hdqt_linear_xent_fwd", X, C.byref(d), X.data_ptr(), W.data_ptr(), labels.data_ptr(), loss.data_ptr(),
          lse.data_ptr(), ws.data_ptr(), nbytes, _status(dev_status, X))
    return loss, lse


def linear_xent_bwd(X, W, labels, lse, g=None, ignore_index: int = -100, reduction: str = "mean", w_is_cd: bool = False,
                    want_dx: bool = True, want_dw: bool = True, piece_bytes: int = 0, dev_status=None):
    """Gradients (dX, dW; None if not wanted) of linear_xent_fwd's loss from its lse.  g: gradient of the loss, an fp32
    scalar (None = 1) or [tokens] with reduction "none".  Works through the vocabulary in pieces of piece_bytes (0 = chosen by
    the library)."""
    X, W, labels, d, ws, nbytes = _xent_call(X, W, labels, ignore_index, reduction, w_is_cd, piece_bytes, XENT_BWD)
    g = _loss_weight(g, reduction, d.tokens, X.device)
    if tuple(lse.shape) != (d.tokens,) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != X.device:
        raise ValueError("lse must be the dense fp32 [tokens] tensor of the forward call")
    dX = torch.empty_like(X, memory_format=torch.contiguous_format) if want_dx else None
    dW = torch.empty_like(W, memory_format=torch.contiguous_format) if want_dw else None
    _call("hdqt_linear_xent_bwd", X, C.byref(d), X.data_ptr(), W.data_ptr(), labels.data_ptr(), lse.data_ptr(),
          _ptr(g), _ptr(dX), _ptr(dW), ws.data_ptr(), nbytes, _status(dev_status, X))
    return dX, dW


def linear_xent_train(X, W, labels, g=None, ignore_index: int = -100, reduction: str = "mean", w_is_cd: bool = False,
                      want_dx: bool = True, want_dw: bool = True, piece_bytes: int = 0, dev_status=None):
    """Loss and gradients in one call (three quarters of the tensor work of linear_xent_fwd + linear_xent_bwd), for a loss whose
    gradient is known beforehand: g as in linear_xent_bwd.  The workspace holds 2 (fp32: 10) bytes per logit of a piece of the
    tokens.  Returns (loss, lse, dX, dW)."""
    X, W, labels, d, ws, nbytes = _xent_call(X, W, labels, ignore_index, reduction, w_is_cd, piece_bytes, XENT_TRAIN)
    g = _loss_weight(g, reduction, d.tokens, X.device)
    lse = X.new_empty(d.tokens, dtype=torch.float32)
    loss = X.new_empty((d.tokens,) if reduction == "none" else (), dtype=torch.float32)
    dX = torch.empty_like(X, memory_format=torch.contiguous_format) if want_dx else None
    dW = torch.empty_like(W, memory_format=torch.contiguous_format) if want_dw else None
    _call("hdqt_linear_xent_train", X, C.byref(d), X.data_ptr(), W.data_ptr(), labels.data_ptr(), _ptr(g),
          loss.data_ptr(), lse.data_ptr(), _ptr(dX), _ptr(dW), ws.data_ptr(), nbytes, _status(dev_status, X))
    return loss, lse, dX, dW
