"""Thin binding over ``libeden.so`` (declared in ``include/eden.h``): ctypes for the sender and
the receiver, the extension ``_binding`` for the calls of the client's training step.

Argument marshalling only: every step of EDEN's sender and receiver, and every product and
checkpoint of the training step, runs in the CUDA kernels of the library.  PyTorch supplies device memory and the stream.  Importing this
module fails loudly if the library has not been built (``python -m
paper_2108_08842_b200.build``); there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, NamedTuple, Optional, Sequence, Union

import numpy as np
import torch

from . import build as _build

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libeden.so")

if not os.path.exists(_LIB_PATH):
    raise ImportError(
        "libeden.so is missing: build it with `python -m paper_2108_08842_b200.build` "
        "(needs nvcc); this package has no CPU fallback")

_lib = ctypes.CDLL(_LIB_PATH)

_u32, _u64, _f64, _vp, _int = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_double, ctypes.c_void_p, ctypes.c_int


class ClientStat(ctypes.Structure):
    _fields_ = [("norm2", _f64), ("dot", _f64), ("received", _f64), ("flags", _u32), ("reserved", _u32)]


def _sig(name, restype, argtypes):
    fn = getattr(_lib, name)
    fn.restype = restype
    fn.argtypes = argtypes
    return fn


_sig("eden_kept_count", _u64, [_u64, _f64])
_sig("eden_rot_dim", _u64, [_u64, _f64])
_sig("eden_code_width", _u32, [_f64])
_sig("eden_code_bytes", _u64, [_u64, _f64])
_sig("eden_num_packets", _u64, [_u64, _f64])
_sig("eden_recv_mask_words", _u64, [_u64, _f64])
_sig("eden_workspace_bytes", _u64, [_u64, _u32])
_sig("eden_host_workspace_bytes", _u64, [_u64, _u32])
_sig("eden_table", _int, [_u32, _vp, _vp])
_sig("eden_pass_plan", _int, [_u64, _f64, _vp, _u32, ctypes.POINTER(_u32)])
_sig("eden_create", _int, [ctypes.POINTER(_vp), _int, _vp, _vp, _u64])
_sig("eden_destroy", _int, [_vp])
_sig("eden_encode", _int, [_vp, _vp, _u64, _u64, _u32, _vp, _vp, _vp, _vp])
_sig("eden_decode_accumulate", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp, _vp])
_sig("eden_mean", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp])
_sig("eden_sparsification_mask", _int, [_vp, _u64, _u64, _f64, _vp])
_sig("eden_encode_host", _int, [_vp, _vp, _u64, _u64, _u32, _vp, _vp, _vp, _vp])
_sig("eden_mean_host", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp])
_sig("eden_status", _int, [_vp, ctypes.POINTER(_u32)])
_sig("eden_client_stats", _int, [_vp, _u32, _vp])
_sig("eden_launch_count", _u64, [_vp])
_sig("eden_sparsification_mask_noalloc", _int, [_int, _vp, _u64, _u64, _f64, _vp])
_sig("eden_strerror", ctypes.c_char_p, [_int])
_sig("eden_mean_partial", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _u64, _vp])
_sig("eden_uniform_entropy", _f64, [_f64])
_sig("eden_uniform_delta", _f64, [_f64])
_sig("eden_uniform_values", _int, [_f64, _vp])
_sig("eden_uniform_index_bytes", _u64, [_u64])
_sig("eden_encode_uniform", _int, [_vp, _vp, _u64, _u64, _u32, _vp, _vp, _vp, _vp])
_sig("eden_decode_accumulate_uniform", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp, _vp])
_sig("eden_mean_uniform", _int, [_vp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp])
_sig("eden_index_histogram", _int, [_vp, _vp, _u64, _u32, _vp])
_sig("eden_profile_enable", _int, [_vp, _int])
_sig("eden_force_generic_kernels", _int, [_vp, _int])
_sig("eden_set_option", _int, [_vp, _int, _int])
_sig("eden_self_check", _int, [])
_sig("eden_mask_threshold_band", _int, [_u64, _u64, _int, _vp, _vp])
_sig("eden_after_kept_count", _u64, [_u64, _f64])
_sig("eden_after_code_bytes", _u64, [_u64, _f64])
_sig("eden_after_workspace_bytes", _u64, [_u64, _u32])
_sig("eden_encode_sparsify_after", _int, [_vp, _vp, _u64, _u64, _u32, _vp, _vp, _vp, _vp])
_sig("eden_mean_sparsify_after", _int, [_vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp])
_sig("eden_decode_accumulate_sparsify_after", _int, [_vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp, _vp])
_sig("eden_checkpoint_groups", _u64, [_u64])
_sig("eden_linear_workspace_bytes", _u64, [_u64, _u64, _u64])
_sig("eden_block_workspace_bytes", _u64, [_u64])
_sig("eden_mx4_workspace_bytes", _u64, [_u64, _u64, _u64])
_sig("eden_profile_collect", _int, [_vp, ctypes.POINTER(_u32)])
_sig("eden_profile_get", _int, [_vp, _u32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(_u64),
                                ctypes.POINTER(_f64), ctypes.POINTER(_f64)])

STATUS_ZERO_VECTOR, STATUS_NONFINITE, STATUS_NO_DATA, STATUS_TIMEOUT, STATUS_SCRATCH = 1, 2, 4, 8, 16
OPT_PLAN_VARIANT, OPT_ROW_STAGING, OPT_SEL_ROUNDS, OPT_SLAB_MIB, OPT_SLAB_STREAMS, OPT_SLAB_SIDES, OPT_SEL_BAND, OPT_SEL_AHEAD = 1, 2, 3, 4, 5, 6, 7, 8
OPT_LINEAR_FORM, OPT_LINEAR_SPLITS = 9, 10
LINEAR_AUTO, LINEAR_PAIR, LINEAR_SINGLE, LINEAR_NARROW, LINEAR_FEW = range(5)
PACKET_COORDS = 1024
UNIFORM_MAX_INDEX = 127
UNIFORM_MIN_DELTA = 0.0625


CHECKPOINT_GROUP = 32


class Checkpoint(NamedTuple):
    """Activations [m, n] in 8 bits: int8 codes [m, n], uint8 exponents [m, ceil(n / 32)]."""
    codes: torch.Tensor
    exps: torch.Tensor


class Norm(NamedTuple):
    """A norm of rows: (v - mean) * rate * weight + bias, weight and bias of the activations' type.
    kind "rms": mean 0, rate = 1 / sqrt(mean(v^2) + eps); "layer": the mean off first."""
    weight: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    kind: str = "rms"
    eps: float = 1e-6


class Joined(NamedTuple):
    """What block_join makes; what was not asked for is None.  Statistics are fp32 [m, 2]: mean and rate."""
    x: Optional[torch.Tensor]
    y: Optional[torch.Tensor]
    after_stats: Optional[torch.Tensor]
    before_stats: Optional[torch.Tensor]


class JoinGradients(NamedTuple):
    """What block_join_backward makes: residual, h and a matrix gate in the activations' type, the
    sums over the rows in fp32; None where there is none or it was left out."""
    residual: Optional[torch.Tensor]
    h: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]
    after_weight: Optional[torch.Tensor]
    after_bias: Optional[torch.Tensor]
    before_weight: Optional[torch.Tensor]
    before_bias: Optional[torch.Tensor]


class Mx4(NamedTuple):
    """A matrix [rows, features] in microscaled 4-bit floating point: uint8 codes [rows, 16 * ceil(features / 32)],
    two a byte, and uint8 exponents [ceil(rows / 128), ceil(features / 256), 1024] in the order that
    include/eden.h gives."""
    codes: torch.Tensor
    exps: torch.Tensor
    features: int


class EdenError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__("eden: %s (%d)" % (_lib.eden_strerror(code).decode(), code))


class _NoBinding:
    """In the extension's place where it cannot be loaded: the sender and the receiver do without
    it, a training call says what is missing."""

    def __init__(self, why):
        self.why = why

    def __getattr__(self, name):
        raise ImportError("eden: the training calls need _binding.so, built for this torch: `python -m "
                          "paper_2108_08842_b200.build` (%s)" % self.why)


try:
    from . import _binding  # built with the library; needs torch loaded
    if getattr(_binding, "built_for", None) != _build.built_for():
        raise ImportError("it was built for %s" % getattr(_binding, "built_for", "something older"))
except ImportError as _e:
    _binding = _NoBinding(_e)
else:
    _binding.bind(*(ctypes.cast(getattr(_lib, name), _vp).value for name in (
        "eden_linear", "eden_checkpoint_save", "eden_checkpoint_restore", "eden_act_backward", "eden_linear_input_grad",
        "eden_linear_weight_grad", "eden_block_join", "eden_block_join_backward", "eden_mx4_quantize", "eden_mx4_restore", "eden_mx4_linear",
        "eden_mx4_linear_input_grad", "eden_mx4_linear_weight_grad")), EdenError, Checkpoint, Mx4)


def _check(rc: int):
    if rc != 0:
        raise EdenError(rc)


# ---------------------------------------------------------------------------- size rules
def kept_count(d: int, bits: float) -> int:
    return int(_lib.eden_kept_count(d, bits))


def rot_dim(d: int, bits: float) -> int:
    return int(_lib.eden_rot_dim(d, bits))


def code_width(bits: float) -> int:
    return int(_lib.eden_code_width(bits))


def code_bytes(d: int, bits: float) -> int:
    return int(_lib.eden_code_bytes(d, bits))


def num_packets(d: int, bits: float) -> int:
    return int(_lib.eden_num_packets(d, bits))


def recv_mask_words(d: int, bits: float) -> int:
    return int(_lib.eden_recv_mask_words(d, bits))


def workspace_bytes(d_max: int, n_batch: int) -> int:
    return int(_lib.eden_workspace_bytes(d_max, n_batch))


def mask_threshold_band(d: int, k: int, tenths: int = 40):
    """eden_mask_threshold_band: (lo, hi) of the band of keys predicted to hold the mask's threshold."""
    lo, hi = ctypes.c_uint32(), ctypes.c_uint32()
    _check(_lib.eden_mask_threshold_band(d, k, tenths, ctypes.byref(lo), ctypes.byref(hi)))
    return int(lo.value), int(hi.value)


def after_kept_count(d: int, bits: float) -> int:
    return int(_lib.eden_after_kept_count(d, bits))


def after_code_bytes(d: int, bits: float) -> int:
    return int(_lib.eden_after_code_bytes(d, bits))


def after_workspace_bytes(d: int, n: int) -> int:
    return int(_lib.eden_after_workspace_bytes(d, n))


def host_workspace_bytes(d: int, n: int) -> int:
    return int(_lib.eden_host_workspace_bytes(d, n))


def checkpoint_groups(features: int) -> int:
    return int(_lib.eden_checkpoint_groups(features))


def linear_workspace_bytes(m: int, n: int, k: int) -> int:
    """Workspace of a Context for the training calls with up to m tokens and n x k weights."""
    return int(_lib.eden_linear_workspace_bytes(m, n, k))


def block_workspace_bytes(n: int) -> int:
    """Workspace of a Context for block_join_backward (and its parts) on rows of n values."""
    return int(_lib.eden_block_workspace_bytes(n))


def mx4_workspace_bytes(m: int, n: int, k: int) -> int:
    """Workspace of a Context for the 4-bit calls with up to m tokens and n x k weights."""
    return int(_lib.eden_mx4_workspace_bytes(m, n, k))


def pass_plan(d: int, bits: float):
    """Index bits transformed by each sweep over HBM for one client (sender order)."""
    buf = (_u32 * 8)()
    n = _u32(0)
    _check(_lib.eden_pass_plan(d, bits, buf, 8, ctypes.byref(n)))
    return list(buf[: n.value])


def table(W: int):
    """(values float32[2^W], boundaries float32[2^W - 1]) the kernels quantise with."""
    c = np.zeros(1 << W, dtype=np.float32)
    b = np.zeros(max((1 << W) - 1, 1), dtype=np.float32)
    _check(_lib.eden_table(W, c.ctypes.data, b.ctypes.data))
    return c, b[: (1 << W) - 1]


def uniform_entropy(delta: float) -> float:
    return float(_lib.eden_uniform_entropy(float(delta)))


def uniform_delta(bits: float) -> float:
    """Delta_b of Section 4.3 (0.0 if outside the supported widths)."""
    return float(_lib.eden_uniform_delta(float(bits)))


def uniform_values(delta: float) -> np.ndarray:
    """float32[128]: the value of each magnitude index, as the kernels use it."""
    v = np.zeros(128, dtype=np.float32)
    _check(_lib.eden_uniform_values(float(delta), v.ctypes.data))
    return v


def uniform_index_bytes(d: int) -> int:
    return int(_lib.eden_uniform_index_bytes(d))


def _f64s(v) -> np.ndarray:
    return np.ascontiguousarray(v, dtype=np.float64)


def _u64s(v) -> np.ndarray:
    return np.ascontiguousarray(v, dtype=np.uint64)


def _ptr_table(tensors: Sequence[Optional[torch.Tensor]]):
    arr = (ctypes.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else t.data_ptr()
    return arr


class Context:
    """One device, one stream, one caller-owned workspace (a torch uint8 tensor)."""

    def __init__(self, device: int = 0, workspace_bytes_: Optional[int] = None,
                 d_max: int = 1 << 20, n_batch: int = 1, stream: Optional[torch.cuda.Stream] = None,
                 host_staging: bool = False):
        if not torch.cuda.is_available():
            raise RuntimeError("eden: no CUDA device; this library has no CPU path")
        self.device = device
        if workspace_bytes_ is None:
            workspace_bytes_ = (host_workspace_bytes if host_staging else workspace_bytes)(d_max, n_batch)
        with torch.cuda.device(device):
            self.stream = stream if stream is not None else torch.cuda.current_stream()
            self.workspace = torch.empty(int(workspace_bytes_) + 256, dtype=torch.uint8, device="cuda:%d" % device)
        base = self.workspace.data_ptr()
        aligned = (base + 255) // 256 * 256
        self._h = _vp()
        self.workspace_bytes = int(workspace_bytes_)
        _check(_lib.eden_create(ctypes.byref(self._h), device, self.stream.cuda_stream,
                                aligned, self.workspace_bytes))
        self._native = None
        if not isinstance(_binding, _NoBinding):
            self._native = _binding.native(self._h.value, device, self.stream.cuda_stream, self.stream.stream_id,
                                           self.stream.device_index, self.stream.device_type)

    def close(self):
        if self._h:
            if self._native is not None:
                _binding.close(self._native)
            _lib.eden_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ sender
    def alloc_codes(self, d: int, bits) -> List[torch.Tensor]:
        return [torch.empty(code_bytes(d, float(b)), dtype=torch.uint8, device="cuda:%d" % self.device)
                for b in bits]

    def encode(self, x: torch.Tensor, bits, seeds, codes: Optional[List[torch.Tensor]] = None,
               scales: Optional[torch.Tensor] = None):
        """eden_encode: x is a CUDA fp32 [n, d] tensor (row stride >= d).  Returns (codes, scales)."""
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
        n, d = x.shape
        bits, seeds = _f64s(bits), _u64s(seeds)
        assert len(bits) == n and len(seeds) == n
        if codes is None:
            codes = self.alloc_codes(d, bits)
        if scales is None:
            scales = torch.empty(n, dtype=torch.float32, device=x.device)
        tab = _ptr_table(codes)
        _check(_lib.eden_encode(self._h, x.data_ptr(), x.stride(0), d, n, bits.ctypes.data,
                                seeds.ctypes.data, tab, scales.data_ptr()))
        return codes, scales

    def encode_uniform(self, x: torch.Tensor, delta, seeds, index: Optional[List[torch.Tensor]] = None,
                       scales: Optional[torch.Tensor] = None):
        """eden_encode_uniform: one int8 index per rotated coordinate.  Returns (index, scales)."""
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
        n, d = x.shape
        delta, seeds = _f64s(delta), _u64s(seeds)
        assert len(delta) == n and len(seeds) == n
        if index is None:
            index = [torch.empty(uniform_index_bytes(d), dtype=torch.int8, device=x.device) for _ in range(n)]
        if scales is None:
            scales = torch.empty(n, dtype=torch.float32, device=x.device)
        _check(_lib.eden_encode_uniform(self._h, x.data_ptr(), x.stride(0), d, n, delta.ctypes.data,
                                        seeds.ctypes.data, _ptr_table(index), scales.data_ptr()))
        return index, scales

    def mean_uniform(self, index, scales, delta, seeds, d: int, recv_masks=None,
                     out: Optional[torch.Tensor] = None):
        if out is None:
            out = torch.empty(d, dtype=torch.float32, device=scales.device)
        return self._decode(_lib.eden_mean_uniform, index, scales, delta, seeds, recv_masks, d, out)

    def decode_accumulate_uniform(self, index, scales, delta, seeds, d: int, acc: torch.Tensor, recv_masks=None):
        used = _u32(0)
        self._decode(_lib.eden_decode_accumulate_uniform, index, scales, delta, seeds, recv_masks, d, acc,
                     extra=(ctypes.byref(used),))
        return int(used.value)

    def index_histogram(self, index, d: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """eden_index_histogram: int32 [n, 256], column v + 128 counts index v."""
        n = len(index)
        if out is None:
            out = torch.empty((n, 256), dtype=torch.int32, device=index[0].device)
        _check(_lib.eden_index_histogram(self._h, _ptr_table(index), d, n, out.data_ptr()))
        return out

    # ------------------------------------------------------------------ receiver
    def _decode(self, fn, codes, scales, bits, seeds, recv_masks, d, out, extra=()):
        n = len(codes)
        bits, seeds = _f64s(bits), _u64s(seeds)
        assert len(bits) == n and len(seeds) == n and scales.is_cuda and scales.dtype == torch.float32
        tab = _ptr_table(codes)
        mtab = None if recv_masks is None else _ptr_table(recv_masks)
        _check(fn(self._h, tab, scales.data_ptr(), bits.ctypes.data, seeds.ctypes.data, mtab,
                  d, n, out.data_ptr(), *extra))
        return out

    def mean(self, codes, scales, bits, seeds, d: int, recv_masks=None, out: Optional[torch.Tensor] = None):
        """eden_mean: (1/n) sum_c x_hat_c as a CUDA fp32 [d] tensor."""
        if out is None:
            out = torch.empty(d, dtype=torch.float32, device=scales.device)
        return self._decode(_lib.eden_mean, codes, scales, bits, seeds, recv_masks, d, out)

    def mean_partial(self, codes, scales, bits, seeds, d: int, n_total: int, recv_masks=None,
                     out: Optional[torch.Tensor] = None):
        """eden_mean_partial: (1/n_total) * sum over the given clients; the partial vectors of
        all GPUs add up to the mean over all n_total senders."""
        if out is None:
            out = torch.empty(d, dtype=torch.float32, device=scales.device)
        n = len(codes)
        bits, seeds = _f64s(bits), _u64s(seeds)
        assert len(bits) == n and len(seeds) == n
        tab = _ptr_table(codes)
        mtab = None if recv_masks is None else _ptr_table(recv_masks)
        _check(_lib.eden_mean_partial(self._h, tab, scales.data_ptr(), bits.ctypes.data, seeds.ctypes.data, mtab,
                                      d, n, int(n_total), out.data_ptr()))
        return out

    def decode_accumulate(self, codes, scales, bits, seeds, d: int, acc: torch.Tensor, recv_masks=None,
                          used_so_far: int = 0):
        """eden_decode_accumulate: acc += sum_c x_hat_c; returns used_so_far + the clients counted."""
        used = _u32(used_so_far)
        self._decode(_lib.eden_decode_accumulate, codes, scales, bits, seeds, recv_masks, d, acc,
                     extra=(ctypes.byref(used),))
        return int(used.value)

    # ------------------------------------------------------------------ sparsification after the rotation
    def encode_sparsify_after(self, x: torch.Tensor, bits, seeds, codes: Optional[List[torch.Tensor]] = None,
                              scales: Optional[torch.Tensor] = None):
        """eden_encode_sparsify_after: b < 1 with the mask over the rotated coordinates."""
        assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
        n, d = x.shape
        bits, seeds = _f64s(bits), _u64s(seeds)
        if codes is None:
            codes = [torch.empty(after_code_bytes(d, float(b)), dtype=torch.uint8, device=x.device) for b in bits]
        if scales is None:
            scales = torch.empty(n, dtype=torch.float32, device=x.device)
        _check(_lib.eden_encode_sparsify_after(self._h, x.data_ptr(), x.stride(0), d, n, bits.ctypes.data,
                                               seeds.ctypes.data, _ptr_table(codes), scales.data_ptr()))
        return codes, scales

    def mean_sparsify_after(self, codes, scales, bits, seeds, d: int, out: Optional[torch.Tensor] = None):
        n = len(codes)
        bits, seeds = _f64s(bits), _u64s(seeds)
        if out is None:
            out = torch.empty(d, dtype=torch.float32, device=scales.device)
        _check(_lib.eden_mean_sparsify_after(self._h, _ptr_table(codes), scales.data_ptr(), bits.ctypes.data,
                                             seeds.ctypes.data, d, n, out.data_ptr()))
        return out

    def decode_accumulate_sparsify_after(self, codes, scales, bits, seeds, d: int, acc: torch.Tensor,
                                         used_so_far: int = 0):
        n = len(codes)
        bits, seeds = _f64s(bits), _u64s(seeds)
        used = _u32(used_so_far)
        _check(_lib.eden_decode_accumulate_sparsify_after(self._h, _ptr_table(codes), scales.data_ptr(),
                                                          bits.ctypes.data, seeds.ctypes.data, d, n,
                                                          acc.data_ptr(), ctypes.byref(used)))
        return int(used.value)

    def sparsification_mask(self, seed: int, d: int, bits: float) -> torch.Tensor:
        """Bitmap (int32 words, bit i of word i/32) of the coordinates kept for b < 1."""
        out = torch.zeros((d + 31) // 32, dtype=torch.int32, device="cuda:%d" % self.device)
        _check(_lib.eden_sparsification_mask(self._h, int(seed), d, float(bits), out.data_ptr()))
        return out

    # ------------------------------------------------------------------ host-buffer variants
    def encode_host(self, x: np.ndarray, bits, seeds, codes: List[np.ndarray], scales: np.ndarray):
        """eden_encode_host: numpy/pinned host buffers in, host buffers out (synchronous)."""
        n, d = x.shape
        bits, seeds = _f64s(bits), _u64s(seeds)
        tab = (ctypes.c_void_p * n)(*[c.ctypes.data for c in codes])
        _check(_lib.eden_encode_host(self._h, x.ctypes.data, x.strides[0] // 4, d, n, bits.ctypes.data,
                                     seeds.ctypes.data, tab, scales.ctypes.data))

    def mean_host(self, codes: List[np.ndarray], scales: np.ndarray, bits, seeds, d: int,
                  recv_masks: Optional[List[Optional[np.ndarray]]], out: np.ndarray):
        n = len(codes)
        bits, seeds = _f64s(bits), _u64s(seeds)
        tab = (ctypes.c_void_p * n)(*[c.ctypes.data for c in codes])
        mtab = None
        if recv_masks is not None:
            mtab = (ctypes.c_void_p * n)(*[None if m is None else m.ctypes.data for m in recv_masks])
        _check(_lib.eden_mean_host(self._h, tab, scales.ctypes.data, bits.ctypes.data, seeds.ctypes.data,
                                   mtab, d, n, out.ctypes.data))

    # ------------------------------------------------------------------ the client's training step
    # Wrong types, shapes, devices or names raise ValueError before anything is launched.
    # Outputs that are not given are made on the context's stream.  No autograd graph is recorded:
    # tensors that require gradients are taken as they are, results require none, and the
    # gradients are those of the calls below.

    def linear(self, x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
               residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, save: str = "none",
               saved: Optional[Checkpoint] = None):
        """eden_linear: act(x [m, k] weight [n, k]^T + bias [n]) + residual [m, n], bf16 or fp16,
        act one of none, relu, gelu, gelu_tanh, silu.  save = "pre" or "out" also returns the
        8-bit checkpoint of the pre-activation or of the result: (out, saved)."""
        return _binding.linear(self._native, x, weight, bias, act, residual, out, save, saved)

    def checkpoint_empty(self, m: int, n: int) -> Checkpoint:
        return _binding.checkpoint_empty(self._native, m, n)

    def checkpoint_save(self, x: torch.Tensor, out: Optional[Checkpoint] = None) -> Checkpoint:
        """eden_checkpoint_save: the 8-bit form of x [m, n] (bf16, fp16 or fp32)."""
        return _binding.checkpoint_save(self._native, x, out)

    def checkpoint_restore(self, saved: Checkpoint, dtype: torch.dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """eden_checkpoint_restore: the values that a checkpoint stands for."""
        return _binding.checkpoint_restore(self._native, saved, dtype, out)

    def act_backward(self, dy: torch.Tensor, pre: Optional[Checkpoint], act: str = "none", out: Union[torch.Tensor, bool, None] = None,
                     bias_grad: Union[torch.Tensor, bool, None] = None, accumulate: bool = False):
        """eden_act_backward: (dz, bias_grad) with dz = dy * act'(pre) and bias_grad its fp32
        column sums (accumulate: added to the given bias_grad).  out=False or bias_grad=False
        leaves that one out: it is neither made nor computed, and None in the result."""
        return _binding.act_backward(self._native, dy, pre, act, out, bias_grad, accumulate)

    def linear_input_grad(self, dz: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None,
                          pre: Optional[Checkpoint] = None, act: str = "none", out: Optional[torch.Tensor] = None,
                          bias_grad: Union[torch.Tensor, bool, None] = None, accumulate: bool = False):
        """eden_linear_input_grad: dx = (dz [m, n] weight [n, k] + residual [m, k]) * act'(pre).
        With pre (the pre-activation of the layer that made the input) or bias_grad given,
        returns (dx, bias_grad), bias_grad the fp32 column sums of dx; else, and with
        bias_grad=False, dx."""
        return _binding.input_grad(self._native, dz, weight, residual, pre, act, out, bias_grad, accumulate)

    def linear_weight_grad(self, dz: torch.Tensor, x, out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """eden_linear_weight_grad: dz [m, n]^T x [m, k] in fp32; x is a Checkpoint or a matrix
        of dz's type (a Checkpoint stands for its values in that type: fp16 saturates and rounds
        what it cannot hold).  out may be a view into the vector that encode takes (accumulate:
        added to what it holds)."""
        return _binding.weight_grad(self._native, dz, x, out, accumulate)

    # ------------------------------------------------------------------ what joins the client's blocks
    def block_join(self, h: torch.Tensor, residual: Optional[torch.Tensor] = None, after: Optional[Norm] = None, before: Optional[Norm] = None,
                   gate: Optional[torch.Tensor] = None, scale: float = 1.0, drop: float = 0.0, seed: Union[int, torch.Tensor] = 0, first_row: int = 0,
                   out: Union[torch.Tensor, bool, None] = None, normed: Optional[torch.Tensor] = None, stats: bool = False) -> Joined:
        """eden_block_join: x = scale * residual + gate * dropout(after(h)) and y = before(x), bf16 or
        fp16 [m, n], every part but h optional.  gate: [n] or [m, n].  drop is the chance of a 0; the
        mask belongs to the seed (a number, or one int64 on the device that is read when the call
        runs, for captured calls) and to first_row + row.  out=False leaves x out; stats: the norms'
        statistics are made, for block_join_backward."""
        return Joined(*_binding.join(self._native, h, residual, after, before, gate, scale, drop, seed, first_row, out, normed, stats))

    def block_join_backward(self, dx: Optional[torch.Tensor], dy: Optional[torch.Tensor], h=None, x=None, after_stats: Optional[torch.Tensor] = None,
                            before_stats: Optional[torch.Tensor] = None, after: Optional[Norm] = None, before: Optional[Norm] = None,
                            gate: Optional[torch.Tensor] = None, scale: float = 1.0, drop: float = 0.0, seed: Union[int, torch.Tensor] = 0, first_row: int = 0,
                            residual: Union[torch.Tensor, bool, None] = None, out: Union[torch.Tensor, bool, None] = None,
                            gate_grad: Union[torch.Tensor, bool, None] = None, after_weight_grad: Union[torch.Tensor, bool, None] = None,
                            after_bias_grad: Union[torch.Tensor, bool, None] = None, before_weight_grad: Union[torch.Tensor, bool, None] = None,
                            before_bias_grad: Union[torch.Tensor, bool, None] = None, accumulate: bool = False) -> JoinGradients:
        """eden_block_join_backward: the gradients of block_join from those of x (dx, or None) and y
        (dy, with a norm before).  h (with a norm after or a gate) and x (with a norm before) are
        matrices or Checkpoints.  An output is made where there is something that it is the gradient
        of, written where it is given, and neither made nor computed where it is False; accumulate:
        the sums over the rows are added to the given ones."""
        return JoinGradients(*_binding.join_backward(self._native, dx, dy, h, x, after_stats, before_stats, after, before, gate, scale, drop, seed, first_row,
                                                     residual, out, gate_grad, after_weight_grad, after_bias_grad, before_weight_grad, before_bias_grad,
                                                     accumulate))

    def norm(self, x: torch.Tensor, norm: Norm, out: Optional[torch.Tensor] = None, stats: bool = False):
        """The norm of x's rows alone; stats: (y, statistics)."""
        j = _binding.join(self._native, x, None, None, norm, None, 1.0, 0.0, 0, 0, False, out, stats)
        return (j[1], j[3]) if stats else j[1]

    def norm_backward(self, dy: torch.Tensor, x, stats: torch.Tensor, norm: Norm, dx: Optional[torch.Tensor] = None,
                      out: Union[torch.Tensor, bool, None] = None, weight_grad: Union[torch.Tensor, bool, None] = None,
                      bias_grad: Union[torch.Tensor, bool, None] = None, accumulate: bool = False):
        """(gradient of x, of the weight, of the bias); x a matrix or a Checkpoint; dx is added to the first."""
        d = _binding.join_backward(self._native, dx, dy, None, x, None, stats, None, norm, None, 1.0, 0.0, 0, 0, False, out, None, None, None,
                                   weight_grad, bias_grad, accumulate)
        return d[1], d[5], d[6]

    def dropout(self, x: torch.Tensor, drop: float, seed: Union[int, torch.Tensor], first_row: int = 0, residual: Optional[torch.Tensor] = None,
                scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """scale * residual + dropout(x).  Its own gradient: dropout(dy) with the same seed."""
        return _binding.join(self._native, x, residual, None, None, None, scale, drop, seed, first_row, out, None, False)[0]

    # ------------------------------------------------------------------ products in 4 bits
    def mx4_empty(self, rows: int, features: int) -> Mx4:
        return _binding.mx4_empty(self._native, rows, features)

    def mx4_quantize(self, x: torch.Tensor, out: Optional[Mx4] = None) -> Mx4:
        """eden_mx4_quantize: the 4-bit form of x [m, n] (bf16, fp16 or fp32), groups along its rows."""
        return _binding.mx4_quantize(self._native, x, out, False)

    def mx4_quantize_transposed(self, x: torch.Tensor, out: Optional[Mx4] = None) -> Mx4:
        """eden_mx4_quantize: the 4-bit form of x^T [n, m], groups along x's columns."""
        return _binding.mx4_quantize(self._native, x, False, out)

    def mx4_quantize_both(self, x: torch.Tensor, rows: Optional[Mx4] = None, columns: Optional[Mx4] = None):
        """Both from one read of x: (mx4_quantize(x), mx4_quantize_transposed(x))."""
        return _binding.mx4_quantize(self._native, x, rows, columns)

    def mx4_restore(self, q: Mx4, dtype: torch.dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """eden_mx4_restore: the values that a 4-bit form stands for."""
        return _binding.mx4_restore(self._native, q, dtype, out)

    def mx4_linear(self, x, weight: Mx4, bias: Optional[torch.Tensor] = None, act: str = "none", residual: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, save: str = "none", saved: Optional[Checkpoint] = None, dtype: Optional[torch.dtype] = None):
        """eden_mx4_linear: `linear` with both operands in 4 bits.  x [m, k] is a matrix (bf16 or
        fp16), which the call quantises, or an Mx4; the rest is then of dtype, else of the type of the
        tensors that are given, else bf16."""
        return _binding.mx4_linear(self._native, x, weight, bias, act, residual, out, save, saved, dtype)

    def mx4_linear_input_grad(self, dz, weight_t: Mx4, residual: Optional[torch.Tensor] = None, pre: Optional[Checkpoint] = None, act: str = "none",
                              out: Optional[torch.Tensor] = None, bias_grad: Union[torch.Tensor, bool, None] = None, accumulate: bool = False,
                              dtype: Optional[torch.dtype] = None):
        """eden_mx4_linear_input_grad: `linear_input_grad` in 4 bits, weight_t = mx4_quantize_transposed(weight)."""
        return _binding.mx4_input_grad(self._native, dz, weight_t, residual, pre, act, out, bias_grad, accumulate, dtype)

    def mx4_linear_weight_grad(self, dz_t: Mx4, x_t: Mx4, out: Optional[torch.Tensor] = None, accumulate: bool = False) -> torch.Tensor:
        """eden_mx4_linear_weight_grad: dz^T x in fp32 from mx4_quantize_transposed of both."""
        return _binding.mx4_weight_grad(self._native, dz_t, x_t, out, accumulate)

    # ------------------------------------------------------------------ status
    def status(self) -> int:
        w = _u32(0)
        _check(_lib.eden_status(self._h, ctypes.byref(w)))
        return int(w.value)

    def client_stats(self, n: int):
        arr = (ClientStat * n)()
        _check(_lib.eden_client_stats(self._h, n, arr))
        return [dict(norm2=a.norm2, dot=a.dot, received=a.received, flags=a.flags) for a in arr]

    def force_generic_kernels(self, on: bool):
        _check(_lib.eden_force_generic_kernels(self._h, 1 if on else 0))

    def set_option(self, option: int, value: int):
        """eden_set_option: one of the OPT_* switches of this module."""
        _check(_lib.eden_set_option(self._h, int(option), int(value)))

    def profile(self, on: bool):
        _check(_lib.eden_profile_enable(self._h, 1 if on else 0))

    def profile_collect(self):
        """Per-kernel totals since profile(True): name -> dict(launches, ms, bytes)."""
        n = _u32(0)
        _check(_lib.eden_profile_collect(self._h, ctypes.byref(n)))
        out = {}
        for i in range(n.value):
            name, launches, ms, nbytes = ctypes.c_char_p(), _u64(0), _f64(0), _f64(0)
            _check(_lib.eden_profile_get(self._h, i, ctypes.byref(name), ctypes.byref(launches),
                                         ctypes.byref(ms), ctypes.byref(nbytes)))
            out[name.value.decode()] = dict(launches=int(launches.value), ms=float(ms.value),
                                            bytes=float(nbytes.value))
        return out

    @property
    def launch_count(self) -> int:
        return int(_lib.eden_launch_count(self._h))


NOALLOC_MAX_DIM = 1 << 24


def sparsification_mask_noalloc(seed: int, d: int, bits: float, out: torch.Tensor,
                                device: int = 0, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """eden_sparsification_mask_noalloc: the b < 1 mask bitmap for callers that cannot
    allocate device memory (no context, no workspace; scratch is a fixed array inside the
    library).  `out` is a caller-owned CUDA int32 tensor of ceil(d/32) words.  Calls that
    overlap on the GPU share that scratch and race; keep them on one stream."""
    assert out.is_cuda and out.dtype == torch.int32 and out.numel() >= (d + 31) // 32
    s = stream if stream is not None else torch.cuda.current_stream(device)
    _check(_lib.eden_sparsification_mask_noalloc(device, s.cuda_stream, int(seed), int(d), float(bits),
                                                 out.data_ptr()))
    return out


# module-level calls with the names of the C entry points ---------------------------------
def eden_encode(ctx: Context, x, bits, seeds, codes=None, scales=None):
    return ctx.encode(x, bits, seeds, codes, scales)


def eden_mean(ctx: Context, codes, scales, bits, seeds, d, recv_masks=None, out=None):
    return ctx.mean(codes, scales, bits, seeds, d, recv_masks, out)


def eden_decode_accumulate(ctx: Context, codes, scales, bits, seeds, d, acc, recv_masks=None):
    return ctx.decode_accumulate(codes, scales, bits, seeds, d, acc, recv_masks)


def eden_encode_uniform(ctx: Context, x, delta, seeds, index=None, scales=None):
    return ctx.encode_uniform(x, delta, seeds, index, scales)


def eden_mean_uniform(ctx: Context, index, scales, delta, seeds, d, recv_masks=None, out=None):
    return ctx.mean_uniform(index, scales, delta, seeds, d, recv_masks, out)


def eden_decode_accumulate_uniform(ctx: Context, index, scales, delta, seeds, d, acc, recv_masks=None):
    return ctx.decode_accumulate_uniform(index, scales, delta, seeds, d, acc, recv_masks)


def eden_index_histogram(ctx: Context, index, d, out=None):
    return ctx.index_histogram(index, d, out)


def eden_mean_partial(ctx: Context, codes, scales, bits, seeds, d, n_total, recv_masks=None, out=None):
    return ctx.mean_partial(codes, scales, bits, seeds, d, n_total, recv_masks, out)


def eden_linear(ctx: Context, x, weight, bias=None, act="none", residual=None, out=None, save="none", saved=None):
    return ctx.linear(x, weight, bias, act, residual, out, save, saved)


def eden_checkpoint_save(ctx: Context, x, out=None):
    return ctx.checkpoint_save(x, out)


def eden_checkpoint_restore(ctx: Context, saved, dtype, out=None):
    return ctx.checkpoint_restore(saved, dtype, out)


def eden_act_backward(ctx: Context, dy, pre, act="none", out=None, bias_grad=None, accumulate=False):
    return ctx.act_backward(dy, pre, act, out, bias_grad, accumulate)


def eden_linear_input_grad(ctx: Context, dz, weight, residual=None, pre=None, act="none", out=None, bias_grad=None, accumulate=False):
    return ctx.linear_input_grad(dz, weight, residual, pre, act, out, bias_grad, accumulate)


def eden_linear_weight_grad(ctx: Context, dz, x, out=None, accumulate=False):
    return ctx.linear_weight_grad(dz, x, out, accumulate)


def eden_block_join(ctx: Context, h, residual=None, after=None, before=None, gate=None, scale=1.0, drop=0.0, seed=0, first_row=0, out=None,
                    normed=None, stats=False):
    return ctx.block_join(h, residual, after, before, gate, scale, drop, seed, first_row, out, normed, stats)


def eden_block_join_backward(ctx: Context, dx, dy, h=None, x=None, after_stats=None, before_stats=None, **rest):
    return ctx.block_join_backward(dx, dy, h, x, after_stats, before_stats, **rest)


def eden_mx4_quantize(ctx: Context, x, rows=None, columns=False):
    """rows, columns: an Mx4 to write, None (made) or False (left out)."""
    return _binding.mx4_quantize(ctx._native, x, rows, columns)


def eden_mx4_restore(ctx: Context, q, dtype, out=None):
    return ctx.mx4_restore(q, dtype, out)


def eden_mx4_linear(ctx: Context, x, weight, bias=None, act="none", residual=None, out=None, save="none", saved=None, dtype=None):
    return ctx.mx4_linear(x, weight, bias, act, residual, out, save, saved, dtype)


def eden_mx4_linear_input_grad(ctx: Context, dz, weight_t, residual=None, pre=None, act="none", out=None, bias_grad=None, accumulate=False, dtype=None):
    return ctx.mx4_linear_input_grad(dz, weight_t, residual, pre, act, out, bias_grad, accumulate, dtype)


def eden_mx4_linear_weight_grad(ctx: Context, dz_t, x_t, out=None, accumulate=False):
    return ctx.mx4_linear_weight_grad(dz_t, x_t, out, accumulate)
