"""Thin ctypes binding over the C ABI declared in ``include/bdr.h``.

Argument marshalling only: torch tensors provide device memory and streams, every step of the
method runs inside the CUDA library.  There is no CPU fallback: if the library is missing, loading
raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbdr_b200.so")

SCALE_POW2, SCALE_FP32_INT, SCALE_FP32_FP, SCALE_FP32_VSQ = 0, 1, 2, 3
ROUND_NEAREST_EVEN, ROUND_NEAREST_AWAY = 0, 1
F32, BF16 = 0, 1
ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2, 3

EXPORTS = ("bdr_strerror", "bdr_device_status", "bdr_packed_sizes", "bdr_quant_dequant", "bdr_pack", "bdr_unpack",
           "bdr_qsnr_workspace_bytes", "bdr_qsnr", "bdr_qsnr_static_max_cfgs", "bdr_qsnr_static", "mx_gemm",
           "mx_gemm_workspace_bytes", "mx_gemm_ws", "mx_gemm_f8_workspace_bytes", "mx_gemm_f8", "bdr_reencode_e4m3", "mx_gemm_e4m3", "bdr_set_workspace",
           "mx_gemm_status", "bdr_selftest_bounded_wait", "bdr_selftest_host", "bdr_qsnr_from_sums", "bdr_pack2", "bdr_qsnr_delayed", "bdr_amax", "bdr_tile_packing_efficiency", "mx_gemm_hw", "bdr_gather_rows", "bdr_device_status_reset", "bdr_quant_dequant_parent",
           "mx_gemv", "mx_kv_append", "mx_attn_decode", "mx_attn_decode_workspace_bytes",
           "mx_gated_gemm", "mx_gated_gemm_workspace_bytes", "mx_gated_gemm_bwd", "mx_gated_gemm_bwd_workspace_bytes", "mx_gated_gemv",
           "mx_cross_entropy", "mx_cross_entropy_workspace_bytes", "mx_cross_entropy_bwd", "mx_cross_entropy_bwd_workspace_bytes")


class BdrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, strerror(status), status))


class _Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k1", "d1", "k2", "d2", "m", "scale_kind", "rounding")]


class _Planes(C.Structure):
    _fields_ = [("exps", C.c_void_p), ("micro", C.c_void_p), ("elems", C.c_void_p),
                ("ld_exps", C.c_int64), ("ld_micro", C.c_int64), ("ld_elems", C.c_int64)]


class _KVCache(C.Structure):
    _fields_ = [("cfg_k", _Config), ("cfg_v", _Config), ("k", _Planes), ("v", _Planes), ("n_pages", C.c_int64),
                ("page_size", C.c_int32), ("n_kv", C.c_int32), ("head_dim", C.c_int32)]


class _Rotation(C.Structure):
    _fields_ = [("cos", C.c_void_p), ("sin", C.c_void_p), ("positions", C.c_void_p), ("ld", C.c_int64), ("n_pos", C.c_int64),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32)]


_ROTATION = struct.Struct("@PPPqqii")  # the same bytes, made once per call


@dataclass(frozen=True)
class Config:
    """bdr_config_t: the (k1, d1, k2, d2, m) tuple of Section III plus scale kind and tie rule."""
    k1: int
    d1: int
    k2: int
    d2: int
    m: int
    scale_kind: int = SCALE_POW2
    rounding: int = ROUND_NEAREST_EVEN

    def c(self) -> _Config:
        try:
            return self._c
        except AttributeError:
            object.__setattr__(self, "_c", _Config(self.k1, self.d1, self.k2, self.d2, self.m, self.scale_kind, self.rounding))
            return self._c


MX9 = Config(16, 8, 2, 1, 7)
MX6 = Config(16, 8, 2, 1, 4)
MX4 = Config(16, 8, 2, 1, 2)


@dataclass
class Planes:
    """Device tensors (uint8, [nlines, ld]) holding the three packed planes."""
    exps: torch.Tensor
    micro: torch.Tensor
    elems: torch.Tensor

    _probe = None

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_probe", None)

    def _describe(self) -> None:
        """Makes the C view, and the calls that tell whether it still holds (a tensor's memory and layout can be exchanged in place)."""
        e, m, x = self.exps, self.micro, self.elems
        probe = (e.data_ptr, m.data_ptr, x.data_ptr, e.stride, m.stride, x.stride)
        view = _Planes(e.data_ptr(), m.data_ptr() if m.numel() else None, x.data_ptr(), e.stride(0), m.stride(0) if m.numel() else 0, x.stride(0))
        sizes = (e.numel, m.numel, x.numel)
        lines = min(t.shape[0] for t in (e, m, x) if t.numel()) if e.numel() else 0
        on_gpu = e.is_cuda and x.is_cuda and (m.is_cuda or not m.numel())
        devices = {t.get_device() for t in (e, m, x) if t.numel()}
        self.__dict__.update(_on_gpu=on_gpu, _device=devices.pop() if on_gpu and len(devices) == 1 else -1, _address=C.addressof(view), _view=view, _known=tuple(f() for f in probe), _probe=probe, _sizes=sizes, _counts=tuple(f() for f in sizes), _lines=lines)

    def lines(self) -> int:
        """Lines that every plane holds."""
        self.c()
        n = self._sizes
        if (n[0](), n[1](), n[2]()) != self._counts:            # cut or extended within its memory
            self._describe()
        return self._lines

    def __reduce__(self):
        return Planes, (self.exps, self.micro, self.elems)

    def c(self) -> _Planes:
        """The C view of the planes.  It is kept from call to call and made again when a plane, or the memory or layout of one, is not
        what it was."""
        p = self._probe
        if p is None or (p[0](), p[1](), p[2](), p[3](), p[4](), p[5]()) != self._known:
            self._describe()
        return self._view


@dataclass
class KVCache:
    """mx_kv_cache_t: a paged key-value cache in MX format.  `k` and `v` are axis-1 planes of [n_pages * page_size,
    n_kv * head_dim] tensors; the object keeps them alive.  Planes and sizes may be replaced, by larger ones for example: the next call
    checks and describes them anew."""
    cfg_k: Config
    cfg_v: Config
    k: Planes
    v: Planes
    n_pages: int
    page_size: int
    n_kv: int
    head_dim: int

    def __post_init__(self):
        self.ref()

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_parts", None)

    def __reduce__(self):
        return KVCache, (self.cfg_k, self.cfg_v, self.k, self.v, self.n_pages, self.page_size, self.n_kv, self.head_dim)

    def _describe(self) -> int:
        for p in (self.k, self.v):
            for t in (p.exps, p.micro, p.elems):
                if t.dtype != torch.uint8 or t.dim() != 2 or t.stride(1) != 1 or t.shape[0] < self.n_pages * self.page_size:
                    raise ValueError("cache planes are uint8 [n_pages * page_size, pitch] tensors")
        k, v = self.k, self.v
        views = k.c(), v.c()
        object.__setattr__(self, "_on_gpu", k._on_gpu and v._on_gpu)
        c = _KVCache(self.cfg_k.c(), self.cfg_v.c(), *views, self.n_pages, self.page_size, self.n_kv, self.head_dim)
        object.__setattr__(self, "_parts", (k, v, k._probe, v._probe, k._known + v._known, C.addressof(c), c))
        return C.addressof(c)

    def ref(self) -> int:
        """Address of the cache's C description, which lives as long as the object and is made again when it does not hold any more."""
        parts = self._parts
        if parts is not None:
            k, v, p, q, known, address, _ = parts
            if k._probe is p and v._probe is q and (p[0](), p[1](), p[2](), p[3](), p[4](), p[5](), q[0](), q[1](), q[2](), q[3](), q[4](), q[5]()) == known:
                return address
        return self._describe()


def alloc_kv_cache(cfg_k: Config, cfg_v: Config, n_pages: int, page_size: int, n_kv: int, head_dim: int, device="cuda") -> KVCache:
    planes = [alloc_planes(cfg, n_pages * page_size, n_kv * head_dim, 1, device) for cfg in (cfg_k, cfg_v)]
    return KVCache(cfg_k, cfg_v, planes[0], planes[1], n_pages, page_size, n_kv, head_dim)


_lib = None


def lib():
    """Load the CUDA library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("CUDA library %s is missing: run paper_2302_08007_b200/build.py "
                              "(or __graft_entry__.build())" % LIB_PATH)
        L = C.CDLL(LIB_PATH)
        L.bdr_strerror.restype = C.c_char_p
        L.bdr_strerror.argtypes = [C.c_int]
        L.bdr_packed_sizes.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_void_p]
        L.bdr_quant_dequant.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64,
                                        C.c_int, C.c_void_p, C.c_void_p]
        L.bdr_pack.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_void_p,
                               C.c_void_p, C.c_void_p, C.c_void_p]
        L.bdr_unpack.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int,
                                 C.c_void_p]
        L.bdr_qsnr_delayed.restype = C.c_int
        L.bdr_qsnr_delayed.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int,
                                       C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.bdr_amax.restype = C.c_int
        L.bdr_amax.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p]
        L.bdr_tile_packing_efficiency.restype = C.c_double
        L.bdr_tile_packing_efficiency.argtypes = [C.c_void_p, C.c_int64, C.c_int64]
        L.mx_gemm_hw.restype = C.c_int
        L.mx_gemm_hw.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_int,
                                 C.c_void_p, C.c_int64, C.c_void_p]
        L.bdr_quant_dequant_parent.restype = C.c_int
        L.bdr_quant_dequant_parent.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64,
                                               C.c_int, C.c_void_p, C.c_void_p]
        L.bdr_gather_rows.restype = C.c_int
        L.bdr_gather_rows.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int,
                                      C.c_int64, C.c_void_p]
        L.bdr_pack2.restype = C.c_int
        L.bdr_pack2.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p,
                                C.c_void_p, C.c_void_p, C.c_void_p]
        L.bdr_qsnr_workspace_bytes.restype = C.c_int64
        L.bdr_qsnr_workspace_bytes.argtypes = [C.c_int]
        L.bdr_qsnr.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int,
                               C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.mx_gemm.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64,
                              C.c_void_p, C.c_int64, C.c_void_p]
        L.bdr_qsnr_static_max_cfgs.restype = C.c_int
        L.bdr_qsnr_static_max_cfgs.argtypes = []
        L.bdr_qsnr_static.restype = C.c_int
        L.bdr_qsnr_static.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int,
                                      C.c_void_p, C.c_void_p]
        L.mx_gemm_workspace_bytes.restype = C.c_int64
        L.mx_gemm_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int64]
        L.mx_gemm_ws.restype = C.c_int
        L.mx_gemm_ws.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64,
                                 C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
        L.mx_gemm_f8_workspace_bytes.restype = C.c_int64
        L.mx_gemm_f8_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int64]
        L.mx_gemm_f8.restype = C.c_int
        L.mx_gemm_f8.argtypes = L.mx_gemm_ws.argtypes
        L.bdr_reencode_e4m3.restype = C.c_int
        L.bdr_reencode_e4m3.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.bdr_set_workspace.restype = C.c_int
        L.bdr_set_workspace.argtypes = [C.c_void_p, C.c_int64]
        L.mx_gemm_e4m3.restype = C.c_int
        L.mx_gemm_e4m3.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_void_p,
                                   C.c_int64, C.c_void_p]
        L.mx_gemm_status.restype = C.c_int
        L.mx_gemm_status.argtypes = []
        L.bdr_device_status.restype = C.c_int
        L.bdr_device_status.argtypes = []
        L.bdr_device_status_reset.restype = C.c_int
        L.bdr_device_status_reset.argtypes = []
        L.bdr_selftest_bounded_wait.restype = C.c_int
        L.bdr_selftest_bounded_wait.argtypes = [C.c_void_p, C.c_void_p]
        L.bdr_selftest_host.restype = C.c_int
        L.bdr_selftest_host.argtypes = []
        L.bdr_qsnr_from_sums.restype = C.c_int
        L.bdr_qsnr_from_sums.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        i32, i64, ptr = C.c_int32, C.c_int64, C.c_void_p
        L.mx_gemv.restype = C.c_int
        L.mx_gemv.argtypes = [ptr, ptr, i64, i64, ptr, C.c_int, i64, i64, ptr, C.c_int, i64, ptr]
        L.mx_kv_append.restype = C.c_int
        L.mx_kv_append.argtypes = [ptr, ptr, i64, ptr, i64, C.c_int, i64, ptr, ptr, ptr, i64, i32, ptr, i64, ptr, ptr, ptr]
        L.mx_attn_decode_workspace_bytes.restype = C.c_int64
        L.mx_attn_decode_workspace_bytes.argtypes = [ptr, i64, i32]
        L.mx_attn_decode.restype = C.c_int
        L.mx_attn_decode.argtypes = [ptr, ptr, i64, C.c_int, i64, i32, ptr, i64, i64, ptr, C.c_float, i32, ptr, i64, ptr, ptr, i64, ptr]
        L.mx_gated_gemv.restype = C.c_int
        L.mx_gated_gemv.argtypes = [ptr, ptr, i64, i64, ptr, C.c_int, i64, i64, i32, ptr, C.c_int, i64, ptr]
        L.mx_gated_gemm_workspace_bytes.restype = i64
        L.mx_gated_gemm_workspace_bytes.argtypes = [i64, i64, i64]
        L.mx_gated_gemm.restype = C.c_int
        L.mx_gated_gemm.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, i32, ptr, C.c_int, i64, ptr, i64, ptr, i64, ptr]
        L.mx_gated_gemm_bwd_workspace_bytes.restype = i64
        L.mx_gated_gemm_bwd_workspace_bytes.argtypes = [i64, i64, i64, C.c_int]
        L.mx_gated_gemm_bwd.restype = C.c_int
        L.mx_gated_gemm_bwd.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, i32, ptr, C.c_int, i64, ptr, i64, ptr, i64, ptr, i64, ptr, i64, ptr]
        L.mx_cross_entropy_workspace_bytes.restype = i64
        L.mx_cross_entropy_workspace_bytes.argtypes = [i64, i64, i64]
        L.mx_cross_entropy.restype = C.c_int
        L.mx_cross_entropy.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, ptr, ptr, ptr, ptr, i64, ptr]
        L.mx_cross_entropy_bwd_workspace_bytes.restype = i64
        L.mx_cross_entropy_bwd_workspace_bytes.argtypes = [i64, i64, i64, C.c_int]
        L.mx_cross_entropy_bwd.restype = C.c_int
        L.mx_cross_entropy_bwd.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, ptr, ptr, ptr, ptr, i64, ptr, i64, C.c_int, ptr, i64, ptr]
        for fn in (L.bdr_packed_sizes, L.bdr_quant_dequant, L.bdr_pack, L.bdr_unpack, L.bdr_qsnr, L.mx_gemm):
            fn.restype = C.c_int
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().bdr_strerror(int(status)).decode()


def _check(status: int, where: str):
    if status != 0:
        raise BdrError(status, where)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("tensor dtype must be float32 or bfloat16")


# The current stream's handle without building a Stream object (3 us of a call that takes 5 in all); torch versions without this
# entry take the ordinary way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _as2d(t: torch.Tensor):
    if t.dim() == 1:
        t = t.unsqueeze(0)
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a 1-D or row-major 2-D tensor")
    return t


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def bdr_packed_sizes(cfg: Config, rows: int, cols: int, axis: int = 1):
    """Default line pitches and plane sizes in bytes: ([ld_exps, ld_micro, ld_elems], [bytes...])."""
    ld = (C.c_int64 * 3)()
    nb = (C.c_int64 * 3)()
    c = cfg.c()
    _check(lib().bdr_packed_sizes(C.addressof(c), rows, cols, axis, C.addressof(ld), C.addressof(nb)),
           "bdr_packed_sizes")
    return list(ld), list(nb)


def alloc_planes(cfg: Config, rows: int, cols: int, axis: int = 1, device="cuda") -> Planes:
    ld, _ = bdr_packed_sizes(cfg, rows, cols, axis)
    nlines = rows if axis == 1 else cols
    mk = lambda l: torch.empty((nlines, l), dtype=torch.uint8, device=device)
    return Planes(mk(ld[0]), mk(ld[1]), mk(ld[2]))


def bdr_quant_dequant(cfg: Config, x: torch.Tensor, y: torch.Tensor | None = None, axis: int = 1,
                      qsnr_sums: torch.Tensor | None = None, stream=None) -> torch.Tensor | None:
    """Q(x) into ``y`` (same dtype/shape/pitch as x; may be x itself).  ``qsnr_sums`` (2 float64 on
    the device) is accumulated into."""
    x2 = _as2d(x)
    y2 = _as2d(y) if y is not None else None
    if y2 is not None and (y2.shape != x2.shape or y2.stride(0) != x2.stride(0) or y2.dtype != x2.dtype):
        raise ValueError("y must match x in shape, pitch and dtype")
    c = cfg.c()
    _check(lib().bdr_quant_dequant(C.addressof(c), _ptr(x2), _ptr(y2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0),
                                   axis, _ptr(qsnr_sums), _stream(stream)), "bdr_quant_dequant")
    return y


def bdr_pack(cfg: Config, x: torch.Tensor, planes: Planes, axis: int = 1, y_dq: torch.Tensor | None = None,
             qsnr_sums: torch.Tensor | None = None, stream=None) -> Planes:
    x2 = _as2d(x)
    y2 = _as2d(y_dq) if y_dq is not None else None
    if y2 is not None and (y2.shape != x2.shape or y2.stride(0) != x2.stride(0) or y2.dtype != x2.dtype):
        raise ValueError("y_dq must match x in shape, pitch and dtype")
    c, p = cfg.c(), planes.c()
    _check(lib().bdr_pack(C.addressof(c), _ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0), axis,
                          C.addressof(p), _ptr(y2), _ptr(qsnr_sums), _stream(stream)), "bdr_pack")
    return planes


def bdr_pack2(cfg: Config, x: torch.Tensor, planes_rows: Planes, planes_cols: Planes, qsnr_sums_rows: torch.Tensor | None = None,
              qsnr_sums_cols: torch.Tensor | None = None, stream=None):
    """Both packed copies of x -- quantized along its rows (axis 1) and along its columns (axis 0) -- from one read."""
    x2 = _as2d(x)
    c, pr, pc = cfg.c(), planes_rows.c(), planes_cols.c()
    _check(lib().bdr_pack2(C.addressof(c), _ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0), C.addressof(pr),
                           C.addressof(pc), _ptr(qsnr_sums_rows), _ptr(qsnr_sums_cols), _stream(stream)), "bdr_pack2")
    return planes_rows, planes_cols


def bdr_quant_dequant_parent(cfg: Config, k_parent: int, x: torch.Tensor, y: torch.Tensor | None, axis: int = 1,
                             qsnr_sums: torch.Tensor | None = None, stream=None):
    """Three-level scaling: FP32 parent scale per k_parent elements of a line above the two-level quantizer (fp32 tensors)."""
    x2 = _as2d(x)
    y2 = _as2d(y) if y is not None else None
    if y2 is not None and (y2.shape != x2.shape or y2.stride(0) != x2.stride(0) or y2.dtype != x2.dtype):
        raise ValueError("y must match x in shape, pitch and dtype")
    c = cfg.c()
    _check(lib().bdr_quant_dequant_parent(C.addressof(c), k_parent, _ptr(x2), _ptr(y2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0),
                                          axis, _ptr(qsnr_sums), _stream(stream)), "bdr_quant_dequant_parent")
    return y


def bdr_gather_rows(cfg: Config, table: Planes, n_rows: int, idx: torch.Tensor, y: torch.Tensor, stream=None) -> torch.Tensor:
    """y[i, :] = decoded row idx[i] of a packed [n_rows, dim] table (axis-1 planes); idx int64 on the device."""
    assert idx.dtype == torch.int64 and idx.is_contiguous() and idx.is_cuda and y.dim() == 2 and y.shape[0] == idx.numel()
    c, p = cfg.c(), table.c()
    _check(lib().bdr_gather_rows(C.addressof(c), C.addressof(p), n_rows, y.shape[1], _ptr(idx), idx.numel(), _ptr(y), _dt(y),
                                 y.stride(0), _stream(stream)), "bdr_gather_rows")
    return y


def bdr_unpack(cfg: Config, planes: Planes, y: torch.Tensor, axis: int = 1, stream=None) -> torch.Tensor:
    y2 = _as2d(y)
    c, p = cfg.c(), planes.c()
    _check(lib().bdr_unpack(C.addressof(c), C.addressof(p), _ptr(y2), _dt(y2), y2.shape[0], y2.shape[1], y2.stride(0),
                            axis, _stream(stream)), "bdr_unpack")
    return y


def bdr_qsnr_workspace_bytes(n_cfgs: int) -> int:
    return int(lib().bdr_qsnr_workspace_bytes(int(n_cfgs)))


def bdr_qsnr(cfgs, x: torch.Tensor, out_db: torch.Tensor, workspace: torch.Tensor, axis: int = 1, stream=None):
    """QSNR in dB of x under every configuration of ``cfgs`` into out_db (float64, len(cfgs))."""
    x2 = _as2d(x)
    arr = (_Config * len(cfgs))(*[c.c() for c in cfgs])
    _check(lib().bdr_qsnr(C.addressof(arr), len(cfgs), _ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0), axis,
                          _ptr(out_db), _ptr(workspace), workspace.numel() * workspace.element_size(),
                          _stream(stream)), "bdr_qsnr")
    return out_db


def bdr_qsnr_delayed(cfgs, x: torch.Tensor, amax_window: torch.Tensor, out_db: torch.Tensor, workspace: torch.Tensor,
                     axis: int = 1, stream=None):
    """bdr_qsnr with the FP32 kinds' first-level maximum taken from `amax_window` (float32 device tensor of earlier
    maxima) instead of from x."""
    assert amax_window.dtype == torch.float32 and amax_window.is_contiguous() and amax_window.is_cuda
    x2 = _as2d(x)
    arr = (_Config * len(cfgs))(*[c.c() for c in cfgs])
    _check(lib().bdr_qsnr_delayed(C.addressof(arr), len(cfgs), _ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0), axis,
                                  _ptr(amax_window), amax_window.numel(), _ptr(out_db), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)), "bdr_qsnr_delayed")
    return out_db


def bdr_amax(x: torch.Tensor, amax: torch.Tensor, stream=None) -> torch.Tensor:
    """amax[0] = max(amax[0], max |x|); amax: one float32 on the device, zeroed by the caller."""
    assert amax.dtype == torch.float32 and amax.numel() == 1 and amax.is_cuda
    x2 = _as2d(x)
    _check(lib().bdr_amax(_ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0), _ptr(amax), _stream(stream)), "bdr_amax")
    return amax


def bdr_tile_packing_efficiency(cfg: Config, tile_elems: int = 256, line_bytes: int = 64) -> float:
    c = cfg.c()
    return float(lib().bdr_tile_packing_efficiency(C.addressof(c), tile_elems, line_bytes))


def bdr_qsnr_static_max_cfgs() -> int:
    return int(lib().bdr_qsnr_static_max_cfgs())


def bdr_qsnr_static(cfgs, x: torch.Tensor, out_db: torch.Tensor, axis: int = 1, stream=None):
    """bdr_qsnr without a workspace argument: the scratch is built into the library, for callers that
    must not allocate device memory (see include/bdr.h).  At most bdr_qsnr_static_max_cfgs()
    configurations; calls that overlap on the GPU race on the shared scratch."""
    x2 = _as2d(x)
    arr = (_Config * len(cfgs))(*[c.c() for c in cfgs])
    _check(lib().bdr_qsnr_static(C.addressof(arr), len(cfgs), _ptr(x2), _dt(x2), x2.shape[0], x2.shape[1], x2.stride(0),
                                 axis, _ptr(out_db), _stream(stream)), "bdr_qsnr_static")
    return out_db


def mx_gemm(cfg_a: Config, a: Planes, cfg_b: Config, b: Planes, M: int, N: int, K: int, c: torch.Tensor, stream=None):
    """c[M,N] (float32) = deq(a)[M,K] @ deq(b)[N,K]^T from packed operands quantized along K."""
    ca, cb, pa, pb = cfg_a.c(), cfg_b.c(), a.c(), b.c()
    _check(lib().mx_gemm(C.addressof(ca), C.addressof(pa), C.addressof(cb), C.addressof(pb), M, N, K, _ptr(c),
                         c.stride(0), _stream(stream)), "mx_gemm")
    return c


def mx_gemm_hw(cfg_a: Config, a: Planes, cfg_b: Config, b: Planes, M: int, N: int, K: int, c: torch.Tensor, r: int = 64, f: int = 25,
               stream=None):
    """c[M,N] (float32) = the product as the dot-product pipeline of Section IV-B computes it (pass length r, f-bit frame)."""
    ca, cb, pa, pb = cfg_a.c(), cfg_b.c(), a.c(), b.c()
    _check(lib().mx_gemm_hw(C.addressof(ca), C.addressof(pa), C.addressof(cb), C.addressof(pb), M, N, K, r, f, _ptr(c),
                            c.stride(0), _stream(stream)), "mx_gemm_hw")
    return c


def mx_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().mx_gemm_workspace_bytes(M, N, K))


def mx_gemm_ws(cfg_a: Config, a: Planes, cfg_b: Config, b: Planes, M: int, N: int, K: int, c: torch.Tensor,
               workspace: torch.Tensor, stream=None):
    """mx_gemm in two phases: decode both operands once into `workspace` (uint8 device tensor of at least
    mx_gemm_workspace_bytes(M, N, K) bytes), then a TMA-fed tensor-core GEMM."""
    ca, cb, pa, pb = cfg_a.c(), cfg_b.c(), a.c(), b.c()
    _check(lib().mx_gemm_ws(C.addressof(ca), C.addressof(pa), C.addressof(cb), C.addressof(pb), M, N, K, _ptr(c),
                            c.stride(0), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "mx_gemm_ws")
    return c


def mx_gemm_f8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().mx_gemm_f8_workspace_bytes(M, N, K))


def mx_gemm_f8(cfg_a: Config, a: Planes, cfg_b: Config, b: Planes, M: int, N: int, K: int, c: torch.Tensor,
               workspace: torch.Tensor, stream=None):
    """mx_gemm for MX4 / MX6 operands on the block-scaled 8-bit tensor-core path: exact re-encoding to E4M3 with
    one scale per 32 elements into `workspace` (at least mx_gemm_f8_workspace_bytes(M, N, K) bytes), then the GEMM."""
    ca, cb, pa, pb = cfg_a.c(), cfg_b.c(), a.c(), b.c()
    _check(lib().mx_gemm_f8(C.addressof(ca), C.addressof(pa), C.addressof(cb), C.addressof(pb), M, N, K, _ptr(c),
                            c.stride(0), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "mx_gemm_f8")
    return c


def bdr_reencode_e4m3(cfg: Config, planes: Planes, rows: int, K: int, out: torch.Tensor, scales: torch.Tensor,
                      inexact: torch.Tensor, stream=None):
    """Packed MX4 / MX6 operand -> E4M3 bytes `out` [rows, K], scale atoms `scales` (rows * K / 32 bytes) and the
    int32 flag `inexact` (set to 1, never cleared, if an element is not representable)."""
    cc, pp = cfg.c(), planes.c()
    _check(lib().bdr_reencode_e4m3(C.addressof(cc), C.addressof(pp), rows, K, _ptr(out), _ptr(scales), _ptr(inexact),
                                   _stream(stream)), "bdr_reencode_e4m3")
    return out, scales


def bdr_set_workspace(workspace: torch.Tensor | None):
    """Lends mx_gemm scratch memory on the current device (None takes it back).  The tensor must stay alive while lent."""
    if workspace is None:
        _check(lib().bdr_set_workspace(None, 0), "bdr_set_workspace")
    else:
        _check(lib().bdr_set_workspace(_ptr(workspace), workspace.numel() * workspace.element_size()), "bdr_set_workspace")


def mx_gemm_e4m3(a: torch.Tensor, scales_a: torch.Tensor, b: torch.Tensor, scales_b: torch.Tensor, M: int, N: int, K: int,
                 c: torch.Tensor, stream=None):
    """C = A B^T from operands re-encoded earlier with bdr_reencode_e4m3 (E4M3 bytes [rows, K] and scale atoms)."""
    _check(lib().mx_gemm_e4m3(_ptr(a), _ptr(scales_a), _ptr(b), _ptr(scales_b), M, N, K, _ptr(c), c.stride(0), _stream(stream)),
           "mx_gemm_e4m3")
    return c


def _pitch(stride: int, rows: int, width: int, what: str) -> int:
    """The pitch of `rows` rows of `width` elements.  With one row at most a stride means nothing; else rows that share memory (an
    expanded view, say) are refused, since a kernel takes a pitch of at least a row."""
    if stride >= width:
        return stride
    if rows > 1:
        raise ValueError("%s: rows share memory (an expanded or overlapping view): make it contiguous" % what)
    return width


def mx_gemv(cfg_w: Config, w: Planes, N: int, K: int, x: torch.Tensor, y: torch.Tensor, stream=None) -> torch.Tensor:
    """y[T,N] = x[T,K] @ deq(w)[N,K]^T for a few rows of x (float32 or bfloat16; y likewise) and weights packed along K."""
    x2, y2 = x if x.dim() == 2 else x.unsqueeze(0), y if y.dim() == 2 else y.unsqueeze(0)
    (T, k), (ldx, sx), (ldy, sy) = x2.shape, x2.stride(), y2.stride()
    lines, c, p = w.lines(), cfg_w.c(), w._view
    if k != K or y2.shape != (T, N) or (sx != 1 and K > 1) or (sy != 1 and N > 1) or lines < N:
        raise ValueError("x is [T, K], y is [T, N], rows contiguous, and the planes hold N lines")
    if not (x.is_cuda and y.is_cuda and w._on_gpu):
        raise ValueError("expected CUDA tensors")
    _check(lib().mx_gemv(C.addressof(c), C.addressof(p), N, K, x2.data_ptr(), _dt(x2), _pitch(ldx, T, K, "x"), T, y2.data_ptr(), _dt(y2),
                         _pitch(ldy, T, N, "y"), _stream(stream)), "mx_gemv")
    return y


def mx_gated_gemv(cfg_w: Config, w: Planes, N: int, K: int, x: torch.Tensor, h: torch.Tensor, act: int = ACT_SILU,
                  stream=None) -> torch.Tensor:
    """h[T,N] = act(x Wg^T) * (x Wu^T) for a few rows of x [T,K] (float32 or bfloat16; h likewise); w is packed [2 N, K], the N
    lines of Wg before those of Wu."""
    x2, h2 = x if x.dim() == 2 else x.unsqueeze(0), h if h.dim() == 2 else h.unsqueeze(0)
    (T, k), (ldx, sx), (ldh, sh) = x2.shape, x2.stride(), h2.stride()
    lines, c, p = w.lines(), cfg_w.c(), w._view
    if k != K or h2.shape != (T, N) or (sx != 1 and K > 1) or (sh != 1 and N > 1) or lines < 2 * N:
        raise ValueError("x is [T, K], h is [T, N], rows contiguous, and the planes hold 2 N lines")
    here = _here()
    if x.get_device() != here or h.get_device() != here or (w._device != here and lines):
        raise ValueError("expected CUDA tensors of the current device")
    _check(lib().mx_gated_gemv(C.addressof(c), C.addressof(p), N, K, x2.data_ptr(), _dt(x2), _pitch(ldx, T, K, "x"), T, act, h2.data_ptr(),
                               _dt(h2), _pitch(ldh, T, N, "h"), _stream(stream)), "mx_gated_gemv")
    return h


def _matrix(t: torch.Tensor, rows: int, cols: int, dtype, what: str, here: int) -> int:
    """Row pitch of a [rows, cols] tensor of `dtype` on the current GPU `here` whose rows are contiguous."""
    if t.shape != (rows, cols) or t.dtype != dtype:
        raise ValueError("%s: expected %s [%d, %d]" % (what, dtype, rows, cols))
    pitch, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: expected contiguous rows" % what)
    if t.get_device() != here:
        raise ValueError("%s: expected a CUDA tensor of the current device" % what)
    return pitch if pitch >= cols else _pitch(pitch, rows, cols, what)


def _vector(t: torch.Tensor, n: int, dtype, what: str, here: int) -> int:
    """Address of a contiguous [n] tensor of `dtype` on the current GPU."""
    if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError("%s: contiguous %s [%d]" % (what, dtype, n))
    if t.get_device() != here:
        raise ValueError("%s: expected a CUDA tensor of the current device" % what)
    return t.data_ptr()


def _operand(p: Planes, lines: int, what: str, here: int) -> int:
    """Address of the C view of planes of at least `lines` lines on the current GPU (Planes.lines and Planes.c in one)."""
    q = p._probe
    if q is None or (q[0](), q[1](), q[2](), q[3](), q[4](), q[5]()) != p._known:
        p._describe()
    n = p._sizes
    if (n[0](), n[1](), n[2]()) != p._counts:
        p._describe()
    if p._lines < lines:
        raise ValueError("%s: the planes hold fewer than %d lines" % (what, lines))
    if p._device != here and lines:
        raise ValueError("%s: expected CUDA tensors of the current device" % what)
    return p._address


def _scratch(t: torch.Tensor, here: int) -> int:
    """Bytes of a workspace."""
    if not t.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    if t.get_device() != here:
        raise ValueError("workspace: expected a CUDA tensor of the current device")
    return t.nbytes


def _here() -> int:
    """The GPU that launches go to; without one no tensor's device equals it."""
    if not torch.cuda.is_initialized():
        if not torch.cuda.is_available():
            return -2
        torch.cuda.init()
    return _raw_device() if _raw_device is not None else torch.cuda.current_device()


def mx_gated_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().mx_gated_gemm_workspace_bytes(M, N, K))


def mx_gated_gemm(cfg_a: Config, a: Planes, cfg_w: Config, w: Planes, M: int, N: int, K: int, h: torch.Tensor, workspace: torch.Tensor,
                  act: int = ACT_SILU, gate_up: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """h[M,N] (float32 or bfloat16) = act(A Wg^T) * (A Wu^T) for A packed [M, K] and w packed [2 N, K], the N lines of Wg before those
    of Wu.  gate_up: [M, 2 N] of h's type for both products, which mx_gated_gemm_bwd reads."""
    here, dtype = _here(), h.dtype
    pa, pw, ldh = _operand(a, M, "a", here), _operand(w, 2 * N, "w", here), _matrix(h, M, N, dtype, "h", here)
    ldg = _matrix(gate_up, M, 2 * N, dtype, "gate_up", here) if gate_up is not None else 0
    ca, cw = cfg_a.c(), cfg_w.c()
    _check(lib().mx_gated_gemm(C.addressof(ca), pa, C.addressof(cw), pw, M, N, K, act, h.data_ptr(), _dt(h), ldh,
                               gate_up.data_ptr() if ldg else None, ldg, workspace.data_ptr(), _scratch(workspace, here), _stream(stream)),
           "mx_gated_gemm")
    return h


def mx_gated_gemm_bwd_workspace_bytes(M: int, N: int, K: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """dtype: of the gradients."""
    return int(lib().mx_gated_gemm_bwd_workspace_bytes(M, N, K, F32 if dtype == torch.float32 else BF16))


def mx_gated_gemm_bwd(cfg_a: Config, a: Planes, cfg_w: Config, w: Planes, M: int, N: int, K: int, dh: torch.Tensor, da: torch.Tensor | None,
                      dw: torch.Tensor | None, workspace: torch.Tensor, act: int = ACT_SILU, gate_up: torch.Tensor | None = None, stream=None):
    """Gradients of mx_gated_gemm from dh [M, N]: da [M, K] and dw [2 N, K] of dh's type (None: not wanted).  gate_up: what the forward
    call stored; None: both products are computed again."""
    here, dtype = _here(), dh.dtype
    pa, pw, ldh = _operand(a, M, "a", here), _operand(w, 2 * N, "w", here), _matrix(dh, M, N, dtype, "dh", here)
    ldg = _matrix(gate_up, M, 2 * N, dtype, "gate_up", here) if gate_up is not None else 0
    lda = _matrix(da, M, K, dtype, "da", here) if da is not None else 0
    ldw = _matrix(dw, 2 * N, K, dtype, "dw", here) if dw is not None else 0
    ca, cw = cfg_a.c(), cfg_w.c()
    _check(lib().mx_gated_gemm_bwd(C.addressof(ca), pa, C.addressof(cw), pw, M, N, K, act, dh.data_ptr(), _dt(dh), ldh,
                                   gate_up.data_ptr() if ldg else None, ldg, da.data_ptr() if lda else None, lda, dw.data_ptr() if ldw else None, ldw,
                                   workspace.data_ptr(), _scratch(workspace, here), _stream(stream)), "mx_gated_gemm_bwd")
    return da, dw


def mx_cross_entropy_workspace_bytes(M: int, V: int, K: int) -> int:
    return int(lib().mx_cross_entropy_workspace_bytes(M, V, K))


def mx_cross_entropy(cfg_a: Config, a: Planes, cfg_w: Config, w: Planes, M: int, V: int, K: int, targets: torch.Tensor, loss: torch.Tensor,
                     lse: torch.Tensor, workspace: torch.Tensor, stream=None):
    """loss and lse (float32 [M]) of the logits A W^T, which are not stored, for A packed [M, K] and w packed [V, K]; targets: int64
    [M], negative = the row does not count (loss 0)."""
    here = _here()
    pa, pw = _operand(a, M, "a", here), _operand(w, V, "w", here)
    t, x, y = _vector(targets, M, torch.int64, "targets", here), _vector(loss, M, torch.float32, "loss", here), _vector(lse, M, torch.float32, "lse", here)
    ca, cw = cfg_a.c(), cfg_w.c()
    _check(lib().mx_cross_entropy(C.addressof(ca), pa, C.addressof(cw), pw, M, V, K, t, x, y, workspace.data_ptr(), _scratch(workspace, here),
                                  _stream(stream)), "mx_cross_entropy")
    return loss, lse


def mx_cross_entropy_bwd_workspace_bytes(M: int, V: int, K: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """dtype: of the gradients."""
    return int(lib().mx_cross_entropy_bwd_workspace_bytes(M, V, K, F32 if dtype == torch.float32 else BF16))


def mx_cross_entropy_bwd(cfg_a: Config, a: Planes, cfg_w: Config, w: Planes, M: int, V: int, K: int, targets: torch.Tensor, lse: torch.Tensor,
                         dloss: torch.Tensor, da: torch.Tensor | None, dw: torch.Tensor | None, workspace: torch.Tensor, stream=None):
    """Gradients of mx_cross_entropy from dloss (float32 [M]) and the forward call's lse: da [M, K] and dw [V, K], both float32 or both
    bfloat16 (None: not wanted)."""
    here = _here()
    pa, pw = _operand(a, M, "a", here), _operand(w, V, "w", here)
    t, x, y = _vector(targets, M, torch.int64, "targets", here), _vector(lse, M, torch.float32, "lse", here), _vector(dloss, M, torch.float32, "dloss", here)
    first = da if da is not None else dw
    dt, dtype = (_dt(first), first.dtype) if first is not None else (F32, None)
    lda = _matrix(da, M, K, dtype, "da", here) if da is not None else 0
    ldw = _matrix(dw, V, K, dtype, "dw", here) if dw is not None else 0
    ca, cw = cfg_a.c(), cfg_w.c()
    _check(lib().mx_cross_entropy_bwd(C.addressof(ca), pa, C.addressof(cw), pw, M, V, K, t, x, y, da.data_ptr() if lda else None, lda,
                                      dw.data_ptr() if ldw else None, ldw, dt, workspace.data_ptr(), _scratch(workspace, here), _stream(stream)),
           "mx_cross_entropy_bwd")
    return da, dw


def _heads(t: torch.Tensor, what: str):
    """Shape and token pitch of a [tokens, heads, head_dim] tensor whose tokens are contiguous."""
    shape = t.shape
    if len(shape) != 3:
        raise ValueError("%s: expected [tokens, heads, head_dim]" % what)
    n, h, d = shape
    if t.is_contiguous():
        return shape, h * d
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != d and h > 1):
        raise ValueError("%s: expected contiguous heads" % what)
    return shape, s0 if s0 >= h * d else _pitch(s0, n, h * d, what)


def mx_kv_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, positions: torch.Tensor | None = None,
                 cos: torch.Tensor | None = None, sin: torch.Tensor | None = None, interleaved: bool = False,
                 q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, k_dq: torch.Tensor | None = None,
                 v_dq: torch.Tensor | None = None, stream=None) -> KVCache:
    """Rotates the keys k [T, n_kv, head_dim] (cos, sin: float32 [n_pos, rot_dim / 2] tables, positions: int64 [T]; None: no
    rotation), quantizes them and v, and writes the lines of `slots` (int64 [T], negative = padding).  Optionally rotates the
    queries q into q_out and returns the quantized values in k_dq / v_dq."""
    shape, ldk = _heads(k, "k")
    vshape, ldv = _heads(v, "v")
    T, dtype = shape[0], k.dtype
    ref = cache.ref()
    if not (k.is_cuda and v.is_cuda and slots.is_cuda and cache._on_gpu):
        raise ValueError("expected CUDA tensors")
    if vshape != shape or shape[1] != cache.n_kv or shape[2] != cache.head_dim or v.dtype != dtype:
        raise ValueError("k and v are [tokens, n_kv, head_dim] of one dtype")
    if slots.dtype != torch.int64 or slots.shape != (T,) or not slots.is_contiguous():
        raise ValueError("slots: contiguous int64 [tokens]")
    rot = None
    if cos is not None:
        if sin is None or positions is None:
            raise ValueError("cos, sin and positions go together")
        if not (cos.is_cuda and sin.is_cuda and positions.is_cuda):
            raise ValueError("expected CUDA tensors")
        (n_pos, half), pitch = cos.shape, cos.stride()
        if cos.dtype != torch.float32 or sin.dtype != torch.float32 or sin.shape != cos.shape or sin.stride() != pitch or (pitch[1] != 1 and half > 1):
            raise ValueError("cos, sin: float32 [n_pos, rot_dim / 2] with one pitch")
        if positions.dtype != torch.int64 or positions.shape != (T,) or not positions.is_contiguous():
            raise ValueError("positions: contiguous int64 [tokens]")
        rot = _ROTATION.pack(cos.data_ptr(), sin.data_ptr(), positions.data_ptr(), _pitch(pitch[0], n_pos, half, "cos, sin"), n_pos, 2 * half, interleaved)
    n_q = ldq = ldo = 0
    if q is not None:
        if q_out is None:
            raise ValueError("q needs q_out")
        if not (q.is_cuda and q_out.is_cuda):
            raise ValueError("expected CUDA tensors")
        (tq, n_q, dq), ldq = _heads(q, "q")
        oshape, ldo = _heads(q_out, "q_out")
        if tq != T or dq != cache.head_dim or oshape != q.shape or q.dtype != dtype or q_out.dtype != dtype:
            raise ValueError("q and q_out are [tokens, n_q, head_dim] of k's dtype")
    for t in (k_dq, v_dq):
        if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda):
            raise ValueError("k_dq, v_dq: contiguous, like k")
    _check(lib().mx_kv_append(ref, k.data_ptr(), ldk, v.data_ptr(), ldv, _dt(k), T, slots.data_ptr(), rot,
                              q.data_ptr() if n_q else None, ldq, n_q, q_out.data_ptr() if n_q else None, ldo,
                              k_dq.data_ptr() if k_dq is not None else None, v_dq.data_ptr() if v_dq is not None else None,
                              _stream(stream)), "mx_kv_append")
    return cache


def mx_attn_decode_workspace_bytes(cache: KVCache, n_seqs: int, n_q: int) -> int:
    return int(lib().mx_attn_decode_workspace_bytes(cache.ref(), n_seqs, n_q))


def mx_attn_decode(cache: KVCache, q: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, out: torch.Tensor,
                   workspace: torch.Tensor, scale: float | None = None, window: int = 0, lse: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """out [B, n_q, head_dim] = attention of one query token per sequence, q [B, n_q, head_dim], over the cached positions
    t < lengths[b] (int32 [B]; the last `window` of them when window > 0) whose pages are page_table[b] (int32 [B, max_pages]).
    lse: float32 [B, n_q].  scale: head_dim ** -0.5 when None."""
    ref = cache.ref()
    if not (q.is_cuda and page_table.is_cuda and lengths.is_cuda and out.is_cuda and workspace.is_cuda and cache._on_gpu):
        raise ValueError("expected CUDA tensors")
    (B, n_q, d), ldq = _heads(q, "q")
    oshape, ldo = _heads(out, "out")
    if d != cache.head_dim or oshape != q.shape or out.dtype != q.dtype:
        raise ValueError("q and out are [sequences, n_q, head_dim] of one dtype")
    (rows, max_pages), (ld_table, step) = page_table.shape, page_table.stride()
    if page_table.dtype != torch.int32 or rows != B or (step != 1 and max_pages > 1):
        raise ValueError("page_table: int32 [sequences, max_pages]")
    if lengths.dtype != torch.int32 or lengths.shape != (B,) or not lengths.is_contiguous():
        raise ValueError("lengths: contiguous int32 [sequences]")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (B, n_q) or not lse.is_contiguous() or not lse.is_cuda):
        raise ValueError("lse: contiguous float32 [sequences, n_q]")
    if not -2 ** 31 <= window < 2 ** 31:                         # as a 32-bit number it would be another one
        if window < 0:
            raise ValueError("window: not negative")
        window = 2 ** 31 - 1                                     # more positions than a cache can have
    _check(lib().mx_attn_decode(ref, q.data_ptr(), ldq, _dt(q), B, n_q, page_table.data_ptr(),
                                _pitch(ld_table, B, max_pages, "page_table"), max_pages, lengths.data_ptr(),
                                d ** -0.5 if scale is None else scale, window, out.data_ptr(), ldo, lse.data_ptr() if lse is not None else None,
                                workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream)), "mx_attn_decode")
    return out


def bdr_device_status() -> int:
    """Sticky per-device status of the kernels' bounded waits (0 = ok); synchronises."""
    return int(lib().bdr_device_status())


def bdr_device_status_reset() -> int:
    """Returns the sticky per-device status word and clears it; synchronises."""
    return int(lib().bdr_device_status_reset())


def bdr_qsnr_from_sums(sums: torch.Tensor, out_db: torch.Tensor, stream=None) -> torch.Tensor:
    """Eq. 3 in dB for every {error, signal} pair of `sums` ([n, 2] or [2] float64, device) into out_db ([n] float64)."""
    assert sums.dtype == torch.float64 and out_db.dtype == torch.float64 and sums.is_contiguous() and out_db.is_contiguous()
    n = sums.numel() // 2
    assert sums.numel() == 2 * n and out_db.numel() >= n
    _check(lib().bdr_qsnr_from_sums(C.c_void_p(sums.data_ptr()), n, C.c_void_p(out_db.data_ptr()), _stream(stream)),
           "bdr_qsnr_from_sums")
    return out_db


def bdr_selftest_bounded_wait(status_word) -> None:
    """Queues the kernel whose bounded wait runs out by design; it leaves BDR_ERR_TIMEOUT (-8) in `status_word`,
    one zeroed int32 on the device."""
    assert status_word.dtype == torch.int32 and status_word.numel() == 1 and status_word.is_cuda
    _check(lib().bdr_selftest_bounded_wait(C.c_void_p(status_word.data_ptr()), _stream(None)), "bdr_selftest_bounded_wait")


def bdr_selftest_host() -> int:
    """Host-only check of the per-device launch bookkeeping and of the cross entropy's pieces (0 = ok); makes no CUDA call."""
    return int(lib().bdr_selftest_host())


def mx_gemm_status() -> int:
    """0, or the (sticky) status of a launch whose bounded device-side wait ran out."""
    return int(lib().mx_gemm_status())
