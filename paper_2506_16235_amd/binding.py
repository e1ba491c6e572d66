"""ctypes binding of libnsml.so -- argument marshalling only.

Same names as the C ABI in include/nsml.h: ``choose_ratio`` (host), ``compress`` and
``decompress`` (GPU, enqueued on torch's current HIP stream), ``payload_layout``.  PyTorch is
used for device memory and streams; every step of the path runs in the library's kernels.
There is no fallback: if the library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Sequence, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnsml.so")

OK, EINVAL, ECAP, EHIP, ENOTIMPL, ENOMEM, EINTERNAL = 0, -1, -2, -3, -4, -5, -6
MAX_KERNELS = 32
CTL_MAX_WIN = 128

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2506_16235_amd.build` "
        "(hipcc, gfx950).  There is no CPU fallback for the GPU path.")

_lib = C.CDLL(LIB_PATH)


class CtlParams(C.Structure):
    _fields_ = [(n, C.c_double) for n in
                ("alpha", "beta1", "beta2", "floor", "cap", "init", "bdp_frac", "rtt_excess",
                 "tr_q", "tr_q4", "tr_d")] + \
               [(n, C.c_int32) for n in ("startup_max", "win_bw", "win_rt", "quant_mode")]


class CtlState(C.Structure):
    _fields_ = [("p", CtlParams), ("ratio", C.c_double), ("btlbw", C.c_double),
                ("rtprop", C.c_double), ("bdp", C.c_double), ("all_max_ebb", C.c_double),
                ("all_min_rtt", C.c_double), ("ebb", C.c_double * CTL_MAX_WIN),
                ("rtt", C.c_double * CTL_MAX_WIN), ("count", C.c_int64), ("phase", C.c_int32),
                ("startup_steps", C.c_int32)]


_vp, _u64, _u32, _i32, _dbl = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int, C.c_double
_lib.nsml_strerror.restype = C.c_char_p
_lib.nsml_strerror.argtypes = [_i32]
_lib.nsml_ctl_default_params.argtypes = [C.POINTER(CtlParams)]
_lib.nsml_ctl_init.argtypes = [C.POINTER(CtlState), C.POINTER(CtlParams)]
_lib.nsml_choose_ratio.argtypes = [C.POINTER(CtlState), _dbl, _dbl, _dbl, _dbl,
                                   C.POINTER(_dbl), C.POINTER(_i32)]
_lib.nsml_payload_layout.argtypes = [_vp, _u32, _dbl, _i32, _u32, _vp, C.POINTER(_u64),
                                     C.POINTER(_u64), C.POINTER(_u64)]
_lib.nsml_create.argtypes = [C.POINTER(_vp), _i32, _u64, _u32, _u32]
_lib.nsml_create_ex.argtypes = [C.POINTER(_vp), _i32, _u64, _u32, _u32, _dbl]
_lib.nsml_create_ex.restype = _i32
_lib.nsml_set_option.argtypes = [_vp, C.c_char_p, _i32]
_lib.nsml_set_option.restype = _i32
_lib.nsml_decompress_static.argtypes = [_vp, _vp, _vp, _u64, _vp, _u32, _dbl, _i32, _u32, _vp, _vp]
_lib.nsml_decompress_static.restype = _i32
_lib.nsml_calibration_stream.argtypes = [_i32, _vp, _vp, _u64, _i32, _vp]
_lib.nsml_calibration_stream.restype = _i32
_lib.nsml_destroy.argtypes = [_vp]
_lib.nsml_last_hip_error.argtypes = [_vp]
_lib.nsml_workspace_bytes.argtypes = [_vp]
_lib.nsml_workspace_bytes.restype = _u64
_lib.nsml_compress.argtypes = [_vp, _vp, _vp, _u64, _vp, _u32, _dbl, _i32, _vp, _vp, _vp, _vp]
_lib.nsml_compress_pruned.argtypes = [_vp, _vp, _vp, _vp, _u64, _vp, _u32, _dbl, _i32, _vp, _vp, _vp, _vp]
_lib.nsml_compress_pruned.restype = _i32
_lib.nsml_decompress.argtypes = [_vp, _vp, _vp, _vp, _u64, _vp, _u32, _dbl, _i32, _vp, _vp]
_lib.nsml_profile_enable.argtypes = [_vp, _i32]
_lib.nsml_profile_read.argtypes = [_vp, _vp, _vp]
_lib.nsml_path_stats.argtypes = [_vp, C.POINTER(_u32), C.POINTER(_u32)]
_lib.nsml_path_stats.restype = _i32
_lib.nsml_bucket_state.argtypes = [_vp, _u32, C.POINTER(_u32)]
_lib.nsml_bucket_state.restype = _i32
_lib.nsml_prune_stats.argtypes = [_vp, C.POINTER(_u32), C.POINTER(_u32)]
_lib.nsml_prune_stats.restype = _i32
_lib.nsml_decompress_accumulate.argtypes = [_vp, _vp, _vp, _vp, _u64, _vp, _u32, _dbl, _i32, _vp, _vp]
_lib.nsml_decompress_accumulate.restype = _i32
_lib.nsml_last_l2norm.argtypes = [_vp, C.POINTER(_dbl), _vp]
_lib.nsml_last_l2norm.restype = _i32
_lib.nsml_calibration_copy.argtypes = [_vp, _vp, _u64, _vp]
_lib.nsml_calibration_copy.restype = _i32
_lib.nsml_kernel_name.argtypes = [_i32]
_lib.nsml_kernel_name.restype = C.c_char_p
for _f in ("nsml_ctl_default_params", "nsml_ctl_init", "nsml_choose_ratio", "nsml_payload_layout",
           "nsml_create", "nsml_destroy", "nsml_last_hip_error", "nsml_compress",
           "nsml_decompress", "nsml_profile_enable", "nsml_profile_read"):
    getattr(_lib, _f).restype = _i32


class NsmlError(RuntimeError):
    def __init__(self, code: int, where: str, hip: int = 0):
        self.code, self.hip = code, hip
        msg = _lib.nsml_strerror(code).decode()
        super().__init__(f"{where}: {msg} (code {code}" + (f", hipError {hip})" if hip else ")"))


def _check(rc: int, where: str, ctx=None):
    if rc != OK:
        hip = _lib.nsml_last_hip_error(ctx) if ctx else 0
        raise NsmlError(rc, where, hip)


def raw():
    """The ctypes library handle (for tests of the C ABI itself)."""
    return _lib


# ----------------------------------------------------------------------- controller

def default_params() -> CtlParams:
    p = CtlParams()
    _check(_lib.nsml_ctl_default_params(C.byref(p)), "nsml_ctl_default_params")
    return p


class Controller:
    """Host-side network-sensing controller state (nsml_ctl_state)."""

    def __init__(self, params: Optional[CtlParams] = None, **overrides):
        p = params or default_params()
        for k, v in overrides.items():
            setattr(p, k, v)
        self.state = CtlState()
        _check(_lib.nsml_ctl_init(C.byref(self.state), C.byref(p)), "nsml_ctl_init")

    def choose_ratio(self, last_payload_bytes: float, last_tx_seconds: float,
                     dense_bytes: float = 0.0, last_l2norm: float = -1.0) -> Tuple[float, int]:
        r, b = _dbl(), _i32()
        _check(_lib.nsml_choose_ratio(C.byref(self.state), last_payload_bytes, last_tx_seconds,
                                      dense_bytes, last_l2norm, C.byref(r), C.byref(b)),
               "nsml_choose_ratio")
        return r.value, b.value


def choose_ratio(ctl: Controller, last_payload_bytes: float, last_tx_seconds: float,
                 dense_bytes: float = 0.0, last_l2norm: float = -1.0) -> Tuple[float, int]:
    return ctl.choose_ratio(last_payload_bytes, last_tx_seconds, dense_bytes, last_l2norm)


# ----------------------------------------------------------------------- geometry

def _off(bucket_off) -> np.ndarray:
    return np.ascontiguousarray(bucket_off, dtype=np.uint64)


def _at(a: np.ndarray) -> int:
    """Address of an array (its ctypes attribute takes 2 us to make)."""
    return a.__array_interface__["data"][0]


def _totals(at: int, buckets: int, ratio: float, bits: int, chunk: int):
    """-> (K, val_bytes, n_scales) of the offsets at an address."""
    K, vb, ns = _u64(), _u64(), _u64()
    rc = _lib.nsml_payload_layout(at, max(buckets, 0), ratio, bits, chunk, None, C.byref(K), C.byref(vb), C.byref(ns))
    if rc != OK:
        _check(rc, "nsml_payload_layout")
    return K.value, vb.value, ns.value


def payload_layout(bucket_off, ratio: float, bits: int, chunk: int = 2048):
    """-> (k_b uint64[B], K, val_bytes, n_scales)."""
    off = _off(bucket_off)
    B = len(off) - 1
    k_b = np.zeros(max(B, 1), dtype=np.uint64)
    K, vb, ns = _u64(), _u64(), _u64()
    _check(_lib.nsml_payload_layout(_at(off), B, ratio, bits, chunk, _at(k_b),
                                    C.byref(K), C.byref(vb), C.byref(ns)), "nsml_payload_layout")
    return k_b[:B], K.value, vb.value, ns.value


# ----------------------------------------------------------------------- GPU path

def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(device: int) -> C.c_void_p:
    """torch's current stream on the device (by index: no Stream object is made)."""
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(device))


def validate_buffers(device, bucket_off, ratio, bits, chunk, *, n=None, grad=None, residual=None,
                     weights=None, idx=None, val=None, scales=None, dense=None):
    """The C ABI carries no capacities, so the sizes, types and placement of every tensor are
    checked here, before a pointer reaches a kernel: a short buffer would be an out-of-bounds
    device write.  Raises ValueError; returns (K, val_bytes, n_scales)."""
    off = _off(bucket_off)
    return _validate(torch.device(device), off, _at(off), ratio, bits, chunk, n, grad, residual, weights, idx, val, scales, dense)


_F32, _INDEX, _BYTES = (torch.float32,), (torch.int32, torch.uint32), (torch.uint8, torch.int8)


def _validate(device, off, at, ratio, bits, chunk, n, grad, residual, weights, idx, val, scales, dense):
    """validate_buffers for offsets as _off gives them, at address `at`."""
    if off.ndim != 1 or len(off) < 2:
        raise ValueError("bucket_off needs at least two entries")
    total = int(off[-1])
    if n is not None and int(n) != total:
        raise ValueError(f"n = {n} but bucket_off ends at {total}")
    K, vb, ns = _totals(at, len(off) - 1, ratio, bits, chunk)

    def want(name, t, dtypes, numel, exact):
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name} must be a torch tensor")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the context is on {device}")
        if t.dtype not in dtypes:
            raise ValueError(f"{name} has dtype {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} is not contiguous")
        have = t.numel()
        if (have != numel) if exact else (have < numel):
            raise ValueError(f"{name} holds {have} elements, needs {'exactly' if exact else 'at least'} {numel}")

    if grad is not None:
        want("grad", grad, _F32, total, True)
    if residual is not None:
        want("residual", residual, _F32, total, True)
    if weights is not None:
        want("weights", weights, _F32, total, True)
    if dense is not None:
        want("dense", dense, _F32, total, True)
    if idx is not None:
        want("idx", idx, _INDEX, K, False)
    if val is not None:
        want("val", val, _BYTES, vb, False)
    if bits <= 8:
        if (idx is not None or val is not None) and scales is None:
            raise ValueError("scales is required for 8- and 4-bit codes")
        if scales is not None:
            want("scales", scales, _F32, ns, False)
    return K, vb, ns


class Context:
    """nsml_ctx: device workspace for gradients of up to max_n elements / max_buckets buckets."""

    # nsml_set_option settings applied to every new context (the tests run the path under each)
    default_options: dict = {}

    def __init__(self, max_n: int, max_buckets: int = 1, chunk: int = 2048, device: int = 0,
                 max_ratio: float = 1.0):
        self.device, self.chunk = int(device), int(chunk)
        self._dev = torch.device("cuda", self.device)
        self._h = _vp()
        rc = _lib.nsml_create_ex(C.byref(self._h), self.device, int(max_n), int(max_buckets), self.chunk,
                                 float(max_ratio))
        if rc != OK:
            raise NsmlError(rc, "nsml_create_ex")
        for name, value in self.default_options.items():
            self.set_option(name, value)

    def set_option(self, name: str, value: int):
        _check(_lib.nsml_set_option(self._h, name.encode(), int(value)), f"nsml_set_option({name})", self._h)

    def close(self):
        if getattr(self, "_h", None):
            _lib.nsml_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def workspace_bytes(self) -> int:
        return int(_lib.nsml_workspace_bytes(self._h))

    def alloc_payload(self, bucket_off, ratio: float, bits: int):
        """Device buffers sized by nsml_payload_layout: (idx, val, scales)."""
        off = _off(bucket_off)
        K, vb, ns = _totals(_at(off), len(off) - 1, ratio, bits, self.chunk)
        dev = self._dev
        idx = torch.empty(K, dtype=torch.int32, device=dev)
        val = torch.empty((vb + 3) // 4 * 4, dtype=torch.uint8, device=dev)
        scales = torch.empty(max(ns, 1), dtype=torch.float32, device=dev)
        return idx, val, scales

    def compress(self, grad: torch.Tensor, residual: torch.Tensor, bucket_off, ratio: float,
                 bits: int, idx: torch.Tensor = None, val: torch.Tensor = None,
                 scales: torch.Tensor = None):
        """nsml_compress on torch's current stream.  residual is updated in place.
        -> (idx int32[K] (bit pattern of uint32), val uint8[...], scales float32[...])."""
        off = _off(bucket_off)
        if idx is None:
            idx, val, scales = self.alloc_payload(off, ratio, bits)
        at = _at(off)
        _validate(self._dev, off, at, ratio, bits, self.chunk, None, grad, residual, None, idx, val, scales, None)
        rc = _lib.nsml_compress(self._h, _ptr(grad), _ptr(residual), grad.numel(), at,
                                len(off) - 1, float(ratio), int(bits), _ptr(idx), _ptr(val),
                                _ptr(scales), _stream(self.device))
        _check(rc, "nsml_compress", self._h)
        return idx, val, scales

    def compress_pruned(self, grad: torch.Tensor, residual: torch.Tensor, weights: torch.Tensor,
                        bucket_off, ratio: float, bits: int, idx: torch.Tensor = None,
                        val: torch.Tensor = None, scales: torch.Tensor = None):
        """nsml_compress_pruned: as compress, after weight-magnitude pruning of the candidates."""
        off = _off(bucket_off)
        if idx is None:
            idx, val, scales = self.alloc_payload(off, ratio, bits)
        at = _at(off)
        _validate(self._dev, off, at, ratio, bits, self.chunk, None, grad, residual, weights, idx, val, scales, None)
        rc = _lib.nsml_compress_pruned(self._h, _ptr(grad), _ptr(residual), _ptr(weights), grad.numel(),
                                       at, len(off) - 1, float(ratio), int(bits),
                                       _ptr(idx), _ptr(val), _ptr(scales), _stream(self.device))
        _check(rc, "nsml_compress_pruned", self._h)
        return idx, val, scales

    def decompress(self, idx: torch.Tensor, val: torch.Tensor, scales: torch.Tensor, n: int,
                   bucket_off, ratio: float, bits: int, out: torch.Tensor = None) -> torch.Tensor:
        off = _off(bucket_off)
        if out is None:
            out = torch.empty(int(n), dtype=torch.float32, device=self._dev)
        at = _at(off)
        _validate(self._dev, off, at, ratio, bits, self.chunk, n, None, None, None, idx, val, scales, out)
        rc = _lib.nsml_decompress(self._h, _ptr(idx), _ptr(val), _ptr(scales), int(n),
                                  at, len(off) - 1, float(ratio), int(bits),
                                  _ptr(out), _stream(self.device))
        _check(rc, "nsml_decompress", self._h)
        return out

    def decompress_accumulate(self, idx, val, scales, bucket_off, ratio: float, bits: int,
                              dense: torch.Tensor) -> torch.Tensor:
        """dense[bucket_off[b] + idx[j]] += decoded value j, in place."""
        off = _off(bucket_off)
        at = _at(off)
        _validate(self._dev, off, at, ratio, bits, self.chunk, None, None, None, None, idx, val, scales, dense)
        rc = _lib.nsml_decompress_accumulate(self._h, _ptr(idx), _ptr(val), _ptr(scales),
                                             dense.numel(), at, len(off) - 1,
                                             float(ratio), int(bits), _ptr(dense), _stream(self.device))
        _check(rc, "nsml_decompress_accumulate", self._h)
        return dense

    def last_l2norm(self, n_buckets: int = 0):
        """-> (norm of the last compressed gradient, per-bucket norms or None).  Synchronises."""
        tot = _dbl()
        per = np.zeros(n_buckets, dtype=np.float64) if n_buckets else None
        _check(_lib.nsml_last_l2norm(self._h, C.byref(tot), _at(per) if n_buckets else None),
               "nsml_last_l2norm", self._h)
        return tot.value, per

    def path_stats(self):
        """-> (fast buckets, fallback buckets) of the last compress call (synchronises)."""
        a, b = _u32(), _u32()
        _check(_lib.nsml_path_stats(self._h, C.byref(a), C.byref(b)), "nsml_path_stats", self._h)
        return a.value, b.value

    def bucket_state(self, b: int):
        """-> dict with the selection state of bucket b after the last compress call (synchronises)."""
        out = (_u32 * 8)()
        _check(_lib.nsml_bucket_state(self._h, b, out), "nsml_bucket_state", self._h)
        names = ("path", "why", "L", "H", "T", "need", "sh", "k")
        return dict(zip(names, (int(x) for x in out)))

    def prune_stats(self):
        """-> (band buckets, dense buckets) of the weight stage of the last compress_pruned (synchronises)."""
        a, b = _u32(), _u32()
        _check(_lib.nsml_prune_stats(self._h, C.byref(a), C.byref(b)), "nsml_prune_stats", self._h)
        return a.value, b.value

    def profile_enable(self, on: bool = True):
        _check(_lib.nsml_profile_enable(self._h, 1 if on else 0), "nsml_profile_enable", self._h)

    def profile_read(self):
        """-> {kernel name: (launches, total ms)} since the last read."""
        n = (C.c_uint32 * MAX_KERNELS)()
        ms = (C.c_double * MAX_KERNELS)()
        _check(_lib.nsml_profile_read(self._h, n, ms), "nsml_profile_read", self._h)
        out = {}
        for i in range(MAX_KERNELS):
            name = _lib.nsml_kernel_name(i)
            if name is not None and n[i]:
                out[name.decode()] = (int(n[i]), float(ms[i]))
        return out


def decompress_accumulate(ctx: Context, idx, val, scales, bucket_off, ratio, bits, dense):
    return ctx.decompress_accumulate(idx, val, scales, bucket_off, ratio, bits, dense)


def decompress_static(idx: torch.Tensor, val: torch.Tensor, scales: Optional[torch.Tensor], n: int, bucket_off,
                      ratio: float, bits: int, chunk: int = 2048, out: torch.Tensor = None) -> torch.Tensor:
    """nsml_decompress_static: decompress without a context and without any allocation inside
    the library (the output tensor is the caller's), on the tensors' device."""
    off = _off(bucket_off)
    dev = idx.device
    if out is None:
        out = torch.empty(int(n), dtype=torch.float32, device=dev)
    at, index = _at(off), dev.index
    _validate(dev, off, at, ratio, bits, chunk, n, None, None, None, idx, val, scales, out)

    def call():
        return _lib.nsml_decompress_static(_ptr(idx), _ptr(val), _ptr(scales), int(n), at, len(off) - 1, float(ratio),
                                           int(bits), int(chunk), _ptr(out), _stream(index))

    if dev.type == "cuda" and torch.cuda.current_device() == index:
        rc = call()
    else:
        with torch.cuda.device(dev):
            rc = call()
    _check(rc, "nsml_decompress_static")
    return out


CALIB_MODES = {"read": 0, "fill": 1, "add": 2, "copy": 3}


def calibration_stream(mode: str, a: torch.Tensor, b: torch.Tensor, nontemporal: bool = False):
    """Plain streaming kernel of the given access pattern over a and b (same byte size)."""
    nbytes = a.numel() * a.element_size()
    assert nbytes == b.numel() * b.element_size()
    _check(_lib.nsml_calibration_stream(CALIB_MODES[mode], _ptr(a), _ptr(b), nbytes, 1 if nontemporal else 0,
                                        _stream(a.device.index)), "nsml_calibration_stream")


def calibration_copy(src: torch.Tensor, dst: torch.Tensor):
    """Plain copy kernel of known size (src -> dst, same byte size, a multiple of 16)."""
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    _check(_lib.nsml_calibration_copy(_ptr(src), _ptr(dst), nbytes, _stream(src.device.index)),
           "nsml_calibration_copy")


def compress(ctx: Context, grad, residual, bucket_off, ratio, bits, idx=None, val=None, scales=None):
    return ctx.compress(grad, residual, bucket_off, ratio, bits, idx, val, scales)


def compress_pruned(ctx: Context, grad, residual, weights, bucket_off, ratio, bits,
                    idx=None, val=None, scales=None):
    return ctx.compress_pruned(grad, residual, weights, bucket_off, ratio, bits, idx, val, scales)


def decompress(ctx: Context, idx, val, scales, n, bucket_off, ratio, bits, out=None):
    return ctx.decompress(idx, val, scales, n, bucket_off, ratio, bits, out)


# ----------------------------------------------------------------------- the 8-bit layer
#
# The gradients are calls of their own, and no result has a graph: tensors that require one are refused while torch records.

Q8_MAX_COLS, NORM_MAX_COLS = 131072, 32768


class _CkptArg(C.Structure):
    _fields_ = [("q", _vp), ("e", _vp), ("ldq", _u64), ("lde", _u64)]


_f32c, _ck = C.c_float, C.POINTER(_CkptArg)
for _name, _args in {
    "nsml_q8_rows": [_vp, _i32, _u64, _u64, _u32, _vp, _vp, _u64, _vp, _vp],
    "nsml_q8_values": [_vp, _u64, _vp, _u64, _u32, _vp, _i32, _u64, _vp],
    "nsml_q8_transpose": [_vp, _u64, _u64, _u32, _vp, _u64, _vp],
    "nsml_q8_matmul": [_vp, _u64, _vp, _vp, _u64, _vp, _vp, _u64, _u32, _u32, _vp, _i32, _u64, _vp],
    "nsml_ckpt8_pack": [_vp, _i32, _u64, _u64, _u32, _ck, _vp],
    "nsml_ckpt8_unpack": [_ck, _u64, _u32, _vp, _i32, _u64, _vp],
    "nsml_ckpt8_wgrad_work": [_u64, _u32, _u32],
    "nsml_ckpt8_wgrad": [_vp, _i32, _u64, _ck, _vp, _u64, _u32, _u32, _vp, _vp, _u64, _vp, _u64, _vp],
    "nsml_rmsnorm_q8": [_vp, _u64, _vp, _u64, _vp, _f32c, _i32, _u64, _u32, _vp, _u64, _vp, _u64, _vp, _vp, _ck, _vp],
    "nsml_rmsnorm_backward_work": [_u64, _u32],
    "nsml_rmsnorm_backward": [_vp, _u64, _ck, _vp, _vp, _vp, _u64, _i32, _u64, _u32, _vp, _u64, _vp, _vp, _u64, _vp],
    "nsml_swiglu_q8": [_vp, _u64, _vp, _u64, _i32, _u64, _u32, _vp, _u64, _vp, _ck, _ck, _ck, _vp],
    "nsml_swiglu_backward": [_vp, _u64, _ck, _ck, _i32, _u64, _u32, _vp, _u64, _vp, _u64, _vp],
}.items():
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = _u64 if _name.endswith("_work") else _i32


class Q8(NamedTuple):
    """A matrix in 8 bits by rows: value = q * scale[row].  q: int8 [rows, cols], its row stride a multiple of 16;
    scale: float32 [rows], or None for 1 (the second operand of q8_matmul only)."""
    q: torch.Tensor
    scale: Optional[torch.Tensor]


class Ckpt8(NamedTuple):
    """A matrix as a checkpoint: value = q * 2 ** (e - 127), one e (uint8 [rows, ceil(cols / 32)]) for 32 neighbours
    of a row.  q as in Q8."""
    q: torch.Tensor
    e: torch.Tensor


class NormQ8(NamedTuple):
    h: torch.Tensor             # x + residual (x itself without a residual)
    y: Q8                       # gamma * h * rstd
    rstd: torch.Tensor          # float32 [rows]
    xhat: Optional[Ckpt8]       # h * rstd


class GluQ8(NamedTuple):
    a: Q8                       # the activation
    gate: Optional[Ckpt8]
    up: Optional[Ckpt8]
    held: Optional[Ckpt8]       # the activation again, for the weight gradient of the product that takes it


_TYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_F32_ONLY, _I8_ONLY, _U8_ONLY = torch.float32, torch.int8, torch.uint8
_recording = torch.is_grad_enabled


def _matrix(name, t, dev, dtype=None, rows=None, cols=None, _Tensor=torch.Tensor):
    """-> (address, elements from row to row, rows, cols) of a matrix whose rows are contiguous."""
    if isinstance(t, _Tensor):
        shape = t.shape
        if len(shape) == 2:
            r, c = shape
            ld, side = t.stride()
            if ((t.dtype in _TYPE if dtype is None else t.dtype is dtype) and t.device == dev and c
                    and (rows is None or r == rows) and (cols is None or c == cols)
                    and (side == 1 or c == 1 or not r) and (ld >= c or r <= 1)
                    and not (t.requires_grad and _recording())):
                return t.data_ptr(), (ld if ld > c else c), r, c
    raise ValueError(_why_not(name, t, dev, dtype, rows, cols))


def _why_not(name, t, dev, dtype, rows, cols) -> str:
    """What _matrix refuses a matrix for."""
    if not isinstance(t, torch.Tensor):
        return f"{name} must be a torch tensor"
    if t.dim() != 2:
        return f"{name} has {t.dim()} dimensions, needs 2"
    if t.device != dev:
        return f"{name} is on {t.device}, not on {dev}"
    if (t.dtype not in _TYPE) if dtype is None else (t.dtype != dtype):
        return f"{name} has dtype {t.dtype}"
    r, c = t.shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        return f"{name} is {r} x {c}, needs {r if rows is None else rows} x {c if cols is None else cols}"
    if c == 0:
        return f"{name} has no columns"
    if t.requires_grad and _recording():
        return _no_graph(name)
    return f"{name} has strides {t.stride()}: rows must be contiguous and must not overlap"


def _no_graph(name) -> str:
    return (f"{name} requires a gradient, and results of the 8-bit layer have no graph: call under torch.no_grad(), "
            "or from the forward of a torch.autograd.Function")


def _vector(name, t, dev, n, _Tensor=torch.Tensor):
    """-> address of a float32 vector, or None."""
    if t is None:
        return None
    if isinstance(t, _Tensor) and t.dtype is _F32_ONLY and t.shape == (n,) and t.device == dev and t.is_contiguous():
        if t.requires_grad and _recording():
            raise ValueError(_no_graph(name))
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous float32 vector of {n} elements on {dev}")


def _codes(name, t, dev, rows=None, cols=None):
    """_matrix of int8 codes: 16-byte aligned rows that own their bytes up to the next multiple of 16."""
    at, ld, r, c = _matrix(name, t, dev, _I8_ONLY, rows, cols)
    if r <= 1:
        ld = (c + 15) & ~15
    if (ld | at) & 15:
        raise ValueError(f"{name}: rows of codes must start at multiples of 16 bytes (strides {t.stride()})")
    if c & 15 and r and t.storage_offset() + (r - 1) * ld + ((c + 15) & ~15) > t.untyped_storage().nbytes():
        raise ValueError(f"{name}: the last row of codes must own its bytes up to the next multiple of 16")
    return at, ld, r, c


def _rows_of(name, x, dev, rows=None, cols=None):
    """-> (address of the codes, ld, rows, cols, address of the scales)."""
    if not isinstance(x, Q8):
        raise ValueError(f"{name} must be a Q8")
    at, ld, r, c = _codes(name + ".q", x.q, dev, rows, cols)
    return at, ld, r, c, _vector(name + ".scale", x.scale, dev, r)


def _ckpt(name, x, dev, rows=None, cols=None):
    """-> (argument, rows, cols) of a checkpoint."""
    if not isinstance(x, Ckpt8):
        raise ValueError(f"{name} must be a Ckpt8")
    at, ld, r, c = _codes(name + ".q", x.q, dev, rows, cols)
    e, lde, _, _ = _matrix(name + ".e", x.e, dev, _U8_ONLY, r, (c + 31) // 32)
    return _CkptArg(at, e, ld, lde), r, c


_int8, _uint8, _float32 = torch.int8, torch.uint8, torch.float32


def _vec(n: int, dtype, dev, _new=torch.empty_strided) -> torch.Tensor:
    """A vector (torch.empty takes 0.7 us longer)."""
    return _new((n,), (1,), dtype=dtype, device=dev)


def _mat(rows: int, cols: int, dtype, dev, _new=torch.empty_strided) -> torch.Tensor:
    return _new((rows, cols), (cols, 1), dtype=dtype, device=dev)


def _new_codes(rows: int, cols: int, dev) -> torch.Tensor:
    """int8 codes whose rows own their bytes up to the next multiple of 16."""
    ld = (cols + 15) & ~15
    q = _mat(rows, ld, _int8, dev)
    return q if ld == cols else q[:, :cols]


def _new_ckpt(rows, cols, dev):
    """-> (Ckpt8, its argument)."""
    q, lde = _new_codes(rows, cols, dev), (cols + 31) >> 5
    e = _mat(rows, lde, _uint8, dev)
    return Ckpt8(q, e), _CkptArg(q.data_ptr(), e.data_ptr(), (cols + 15) & ~15, lde)


def _device_of(name, t) -> torch.device:
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{name} must be a tensor on a GPU")
    return t.device


def _device_of_codes(name, x, kind) -> torch.device:
    if not isinstance(x, kind):
        raise ValueError(f"{name} must be a {kind.__name__}")
    return _device_of(name + ".q", x.q)


def _same_type(name, out, dtype):
    if isinstance(out, torch.Tensor) and out.dtype != dtype:
        raise ValueError(f"{name} has dtype {out.dtype}, not {dtype}")


_written = torch.autograd.graph.increment_version       # torch does not see that the library writes a tensor of the caller's


def _result(name, out, rows, cols, dtype, dev):
    """-> (matrix to write, address, elements from row to row): the caller's, or a new one."""
    if out is None:
        if dtype not in _TYPE:
            raise ValueError(f"results are float32, bfloat16 or float16, not {dtype}")
        out = _mat(rows, cols, dtype, dev)
        return out, out.data_ptr(), cols
    at, ld, _, _ = _matrix(name, out, dev, None, rows, cols)
    _written(out)
    return out, at, ld


_current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _enqueue(dev, fn, *args):
    """One call of the library on torch's current stream of the device."""
    index = dev.index
    if _current_device() == index:
        rc = fn(*args, _current_stream(index))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _current_stream(index))
    if rc != OK:
        _check(rc, fn.__name__)


def q8_rows(x: torch.Tensor, col_scale: Optional[torch.Tensor] = None, out: Optional[Q8] = None) -> Q8:
    """The rows of x (times col_scale by columns) in 8 bits: weights by output channel, tokens."""
    dev = _device_of("x", x)
    at, ld, m, k = _matrix("x", x, dev)
    col = _vector("col_scale", col_scale, dev, k)
    if out is None:
        out = Q8(_new_codes(m, k, dev), _vec(m, _float32, dev))
        q, ldq, s = out.q.data_ptr(), (k + 15) & ~15, out.scale.data_ptr()
    else:
        q, ldq, _, _, s = _rows_of("out", out, dev, m, k)
        if s is None:
            raise ValueError("out.scale is required")
        _written(out)
    _enqueue(dev, _lib.nsml_q8_rows, at, _TYPE[x.dtype], ld, m, k, col, q, ldq, s)
    return out


def q8_transposed(w: Q8) -> Q8:
    """The codes of w the other way round, without scales: what the gradient of the data is multiplied by,
    q8_matmul(q8_rows(dc, col_scale=w.scale), q8_transposed(w)).  A layout to make once per update of the weights."""
    dev = _device_of_codes("w", w, Q8)
    q, ldq, n, k, _ = _rows_of("w", w, dev)
    out = _new_codes(k, n, dev)
    _enqueue(dev, _lib.nsml_q8_transpose, q, ldq, n, k, out.data_ptr(), (n + 15) & ~15)
    return Q8(out, None)


def q8_values(x: Q8, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that 8-bit rows stand for."""
    dev = _device_of_codes("x", x, Q8)
    q, ldq, m, k, s = _rows_of("x", x, dev)
    out, at, ld = _result("out", out, m, k, dtype, dev)
    _enqueue(dev, _lib.nsml_q8_values, q, ldq, s, m, k, at, _TYPE[out.dtype], ld)
    return out


def q8_matmul(a: Q8, b: Q8, dtype: torch.dtype = torch.bfloat16, bias: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a (m x k) times b (n x k, weights by output channel) transposed, plus bias (float32 [n]); the sum is exact."""
    dev = _device_of_codes("a", a, Q8)
    qa, lda, m, k, sa = _rows_of("a", a, dev)
    qb, ldb, n, _, sb = _rows_of("b", b, dev, None, k)
    if sa is None:
        raise ValueError("a.scale is required")
    v = _vector("bias", bias, dev, n)
    out, at, ld = _result("out", out, m, n, dtype, dev)
    _enqueue(dev, _lib.nsml_q8_matmul, qa, lda, sa, qb, ldb, sb, v, m, n, k, at, _TYPE[out.dtype], ld)
    return out


def ckpt8_pack(x: torch.Tensor, out: Optional[Ckpt8] = None) -> Ckpt8:
    """x as a checkpoint in 8 bits."""
    dev = _device_of("x", x)
    at, ld, m, k = _matrix("x", x, dev)
    if out is None:
        out, arg = _new_ckpt(m, k, dev)
    else:
        arg = _ckpt("out", out, dev, m, k)[0]
        _written(out)
    _enqueue(dev, _lib.nsml_ckpt8_pack, at, _TYPE[x.dtype], ld, m, k, arg)
    return out


def ckpt8_unpack(x: Ckpt8, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that a checkpoint stands for."""
    dev = _device_of_codes("x", x, Ckpt8)
    arg, m, k = _ckpt("x", x, dev)
    out, at, ld = _result("out", out, m, k, dtype, dev)
    _enqueue(dev, _lib.nsml_ckpt8_unpack, arg, m, k, at, _TYPE[out.dtype], ld)
    return out


def ckpt8_wgrad(dy: torch.Tensor, x: Ckpt8, col_scale: Optional[torch.Tensor] = None,
                add: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """float32 [n, k]: add + col_scale * (dy transposed times x).  out may be a view of the flat gradient that compress
    takes, and may be add (a sum over micro-batches)."""
    dev = _device_of("dy", dy)
    at, ld, m, n = _matrix("dy", dy, dev)
    arg, _, k = _ckpt("x", x, dev, m)
    col = _vector("col_scale", col_scale, dev, k)
    _same_type("out", out, _float32)
    out, w, ldw = _result("out", out, n, k, _float32, dev)
    base = None
    if add is not None:
        base, lda, _, _ = _matrix("add", add, dev, _F32_ONLY, n, k)
        if n == 1:
            lda = ldw
        if lda != ldw:
            raise ValueError("add and out must have the same row stride")
    need = _lib.nsml_ckpt8_wgrad_work(m, n, k)
    work = _vec(need, _uint8, dev) if need else None
    _enqueue(dev, _lib.nsml_ckpt8_wgrad, at, _TYPE[dy.dtype], ld, arg, col, m, n, k, base, w, ldw,
             None if work is None else work.data_ptr(), need)
    return out


def rmsnorm_q8(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, eps: float = 1e-5,
               residual: Optional[torch.Tensor] = None, checkpoint: bool = False) -> NormQ8:
    """RMS norm of x (+ residual) with its output in 8 bits; checkpoint: the normalized values for the backward pass."""
    dev = _device_of("x", x)
    at, ld, m, k = _matrix("x", x, dev)
    h, r, ldr, ha, ldh = x, None, 0, None, 0
    if residual is not None:
        r, ldr, _, _ = _matrix("residual", residual, dev, x.dtype, m, k)
        h = _mat(m, k, x.dtype, dev)
        ha, ldh = h.data_ptr(), k
    g = _vector("gamma", gamma, dev, k)
    q, scale = _new_codes(m, k, dev), _vec(m, _float32, dev)
    rstd = _vec(m, _float32, dev)
    xhat, arg = _new_ckpt(m, k, dev) if checkpoint else (None, None)
    _enqueue(dev, _lib.nsml_rmsnorm_q8, at, ld, r, ldr, g, eps, _TYPE[x.dtype], m, k, ha, ldh, q.data_ptr(),
             (k + 15) & ~15, scale.data_ptr(), rstd.data_ptr(), arg)
    return NormQ8(h, Q8(q, scale), rstd, xhat)


def rmsnorm_backward(dy: torch.Tensor, xhat: Ckpt8, rstd: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                     dres: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     dgamma: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """-> (gradient of x and of the residual, gradient of gamma).  dres: what reaches the sum by the residual stream."""
    dev = _device_of("dy", dy)
    at, ld, m, k = _matrix("dy", dy, dev)
    arg, _, _ = _ckpt("xhat", xhat, dev, m, k)
    rs, g = _vector("rstd", rstd, dev, m), _vector("gamma", gamma, dev, k)
    if rs is None:
        raise ValueError("rstd is required")
    d, ldd = None, 0
    if dres is not None:
        d, ldd, _, _ = _matrix("dres", dres, dev, dy.dtype, m, k)
    _same_type("out", out, dy.dtype)
    out, o, ldo = _result("out", out, m, k, dy.dtype, dev)
    if dgamma is None:
        dgamma = _vec(k, _float32, dev)
        dg = dgamma.data_ptr()
    else:
        dg = _vector("dgamma", dgamma, dev, k)
        _written(dgamma)
    need = _lib.nsml_rmsnorm_backward_work(m, k)
    work = _vec(need, _uint8, dev)
    _enqueue(dev, _lib.nsml_rmsnorm_backward, at, ld, arg, rs, g, d, ldd, _TYPE[dy.dtype], m, k, o, ldo, dg, work.data_ptr(), need)
    return out, dgamma


def swiglu_q8(gate: torch.Tensor, up: torch.Tensor, checkpoint: bool = False) -> GluQ8:
    """gate / (1 + exp(-gate)) * up in 8 bits by rows; checkpoint: gate, up and the result for the backward pass."""
    dev = _device_of("gate", gate)
    g, ldg, m, k = _matrix("gate", gate, dev)
    u, ldu, _, _ = _matrix("up", up, dev, gate.dtype, m, k)
    q, scale = _new_codes(m, k, dev), _vec(m, _float32, dev)
    held, args = zip(*(_new_ckpt(m, k, dev) for _ in range(3))) if checkpoint else ((None,) * 3,) * 2
    _enqueue(dev, _lib.nsml_swiglu_q8, g, ldg, u, ldu, _TYPE[gate.dtype], m, k, q.data_ptr(), (k + 15) & ~15,
             scale.data_ptr(), *args)
    return GluQ8(Q8(q, scale), *held)


def swiglu_backward(da: torch.Tensor, gate: Ckpt8, up: Ckpt8, dgate: Optional[torch.Tensor] = None,
                    dup: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """-> gradients of gate and up.  dgate and dup may be halves of one matrix."""
    dev = _device_of("da", da)
    at, ld, m, k = _matrix("da", da, dev)
    kg, ku = _ckpt("gate", gate, dev, m, k)[0], _ckpt("up", up, dev, m, k)[0]
    _same_type("dgate", dgate, da.dtype)
    _same_type("dup", dup, da.dtype)
    dgate, g, ldg = _result("dgate", dgate, m, k, da.dtype, dev)
    dup, u, ldu = _result("dup", dup, m, k, da.dtype, dev)
    _enqueue(dev, _lib.nsml_swiglu_backward, at, ld, kg, ku, _TYPE[da.dtype], m, k, g, ldg, u, ldu)
    return dgate, dup
