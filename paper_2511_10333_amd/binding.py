"""ctypes binding with the same names as the C ABI (``include/edgc.h``).

Argument marshalling only: every step of the path runs inside the library's
kernels.  There is no fallback: if ``libedgc.so`` is missing or fails to load,
importing a symbol from it raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import List, Optional, Sequence

F32, BF16 = 0, 1
OK, EINVAL, ENOMEM, EHIP, ENOTIMPL, ENONFINITE = 0, -1, -2, -3, -4, -5

_HERE = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_HERE, "libedgc.so")


class EdgcError(RuntimeError):
    def __init__(self, code: int, what: str, detail: str = ""):
        super().__init__(f"{what}: edgc status {code}" + (f" ({detail})" if detail else ""))
        self.code = code


class _EntropyResult(C.Structure):
    _fields_ = [("H_bits", C.c_double), ("h_diff_nats", C.c_double), ("lo", C.c_float),
                ("hi", C.c_float), ("n_sampled", C.c_uint64), ("n_nonfinite", C.c_uint64),
                ("status", C.c_int32), ("_pad", C.c_int32)]


class _RankParams(C.Structure):
    _fields_ = [("m", C.c_uint32), ("n", C.c_uint32), ("r_min", C.c_uint32), ("r_max", C.c_uint32),
                ("step_limit", C.c_uint32), ("allowed", C.POINTER(C.c_uint32)),
                ("n_allowed", C.c_uint32), ("eta", C.c_double), ("total_iters", C.c_uint64),
                ("min_warmup_frac", C.c_double), ("r_ref", C.c_uint32)]


class _RankState(C.Structure):
    _fields_ = [("have_ref", C.c_int32), ("compressing", C.c_int32), ("H_ref", C.c_double),
                ("r_prev", C.c_double), ("iters_seen", C.c_uint64)]


class _RankDecision(C.Structure):
    _fields_ = [("rank", C.c_uint32), ("_pad", C.c_uint32), ("r_unclamped", C.c_double),
                ("H_mean", C.c_double), ("T_com", C.c_double)]


class _KernelStat(C.Structure):
    _fields_ = [("kernel", C.c_char_p), ("launches", C.c_uint64), ("total_ms", C.c_double),
                ("bytes", C.c_double), ("flops", C.c_double), ("event_overhead_ms", C.c_double)]


ENTROPY_RESULT_BYTES = C.sizeof(_EntropyResult)

_lib: Optional[C.CDLL] = None


def load_library() -> C.CDLL:
    """Loads the in-tree ``libedgc.so``; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    L = C.CDLL(path)
    u64, u32, vp, i32 = C.c_uint64, C.c_uint32, C.c_void_p, C.c_int
    L.edgc_create.restype = i32
    L.edgc_create.argtypes = [C.POINTER(vp), i32, u32, u32, u64, u64]
    L.edgc_destroy.restype = i32
    L.edgc_destroy.argtypes = [vp]
    L.edgc_last_error.restype = C.c_char_p
    L.edgc_last_error.argtypes = [vp]
    L.edgc_profile_begin.restype = i32
    L.edgc_profile_begin.argtypes = [vp, u32]
    L.edgc_profile_end.restype = i32
    L.edgc_profile_end.argtypes = [vp, C.POINTER(_KernelStat), u32, C.POINTER(u32)]
    L.edgc_entropy_estimate.restype = i32
    L.edgc_entropy_estimate.argtypes = [vp, vp, i32, u64, u64, u32, u64, u64, u32, vp, vp, vp, vp]
    L.edgc_entropy_estimate_noalloc.restype = i32
    L.edgc_entropy_estimate_noalloc.argtypes = [vp, vp, i32, u64, u64, u32, u64, u64, u32, vp, vp, vp, vp]
    L.edgc_entropy_estimate_batch.restype = i32
    L.edgc_entropy_estimate_batch.argtypes = [vp, C.POINTER(C.c_void_p), C.POINTER(u64), u32, i32, u64, u32,
                                              u64, u64, u32, vp, vp, vp, vp]
    L.edgc_sample_indices.restype = i32
    L.edgc_sample_indices.argtypes = [vp, u64, u64, u32, u64, u64, vp, u64, C.POINTER(u64), vp]
    L.edgc_select_rank.restype = i32
    L.edgc_select_rank.argtypes = [C.POINTER(_RankState), vp, u32, u64, C.POINTER(_RankParams),
                                   C.POINTER(_RankDecision)]
    L.edgc_rank_bounds.restype = i32
    L.edgc_rank_bounds.argtypes = [C.POINTER(_RankCost), u32, C.c_double, C.c_double, C.c_double,
                                   C.POINTER(_RankBounds), C.POINTER(C.c_double)]
    L.edgc_fit_eta.restype = i32
    L.edgc_fit_eta.argtypes = [C.POINTER(u32), C.POINTER(C.c_double), u32, C.POINTER(C.c_double),
                               C.POINTER(C.c_double)]
    L.edgc_stage_ranks.restype = i32
    L.edgc_stage_ranks.argtypes = [u32, C.c_double, C.c_double, u32, u32, C.POINTER(u32), u32, u32,
                                   C.POINTER(u32), C.POINTER(C.c_double)]
    L.edgc_entropy_due.restype = i32
    L.edgc_entropy_due.argtypes = [u64, u32]
    L.edgc_measure_rank_costs.restype = i32
    L.edgc_measure_rank_costs.argtypes = [vp, vp, i32, u32, u32, u64, vp, vp, u32, vp, u32, vp,
                                          C.POINTER(u32), u32, u32, i32, C.POINTER(_RankCost), vp]
    L.edgc_measure_device_peaks.restype = i32
    L.edgc_measure_device_peaks.argtypes = [vp, vp, vp, u64, u32, C.POINTER(_DevicePeaks), vp]
    L.edgc_tensor_bypassed.restype = i32
    L.edgc_tensor_bypassed.argtypes = [u32, u32, u32]
    L.edgc_reserve_batch.restype = i32
    L.edgc_reserve_batch.argtypes = [vp, C.POINTER(u32), C.POINTER(u32), u32]
    L.edgc_compress_batch.restype = i32
    L.edgc_compress_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, u32, vp]
    L.edgc_decompress_batch.restype = i32
    L.edgc_decompress_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, vp]
    L.edgc_compress_p_batch.restype = i32
    L.edgc_compress_p_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, vp]
    L.edgc_compress_q_batch.restype = i32
    L.edgc_compress_q_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, vp]
    L.edgc_residual_materialize_batch.restype = i32
    L.edgc_residual_materialize_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, vp]
    L.edgc_init_q.restype = i32
    L.edgc_init_q.argtypes = [vp, vp, u32, u32, u32, u32, u64, vp]
    L.edgc_compress.restype = i32
    L.edgc_compress.argtypes = [vp, vp, i32, u32, u32, u64, vp, i32, vp, u32, vp, u32, u32, u32, vp]
    L.edgc_decompress.restype = i32
    L.edgc_decompress.argtypes = [vp, vp, u32, vp, u32, u32, u32, u32, vp, vp, i32, u64, vp]
    f32 = C.c_float
    L.edgc_grad_sumsq_batch.restype = i32
    L.edgc_grad_sumsq_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, i32, vp, vp]
    L.edgc_clip_batch.restype = i32
    L.edgc_clip_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, C.c_double, vp, vp, vp]
    L.edgc_reserve_block_norm.restype = i32
    L.edgc_reserve_block_norm.argtypes = [vp, u32, u32]
    L.edgc_block_norm_forward.restype = i32
    L.edgc_block_norm_forward.argtypes = [vp, i32, u64, u32, vp, vp, vp, vp, u64, vp, f32, f32, vp, vp, vp, vp, vp]
    L.edgc_block_norm_backward.restype = i32
    L.edgc_block_norm_backward.argtypes = [vp, i32, u64, u32, vp, vp, vp, vp, vp, vp, u64, vp, vp, vp, f32, vp, vp, vp, vp,
                                           vp, vp]
    L.edgc_reserve_ff.restype = i32
    L.edgc_reserve_ff.argtypes = [vp, i32, u32, u32, u32, i32]
    L.edgc_ff_forward.restype = i32
    L.edgc_ff_forward.argtypes = [vp, C.POINTER(_FF), vp, u64, u32, vp, u64, vp, vp, u64, vp]
    L.edgc_ff_backward.restype = i32
    L.edgc_ff_backward.argtypes = [vp, C.POINTER(_FF), vp, u64, u32, vp, vp, u64, vp, u64, vp, u64, vp, u64, vp, u64, vp, u64, i32, vp]
    f64 = C.c_double
    L.edgc_reserve_orthogonalize.restype = i32
    L.edgc_reserve_orthogonalize.argtypes = [vp, i32, C.POINTER(u32), C.POINTER(u32), u32, u32]
    L.edgc_orthogonalize_batch.restype = i32
    L.edgc_orthogonalize_batch.argtypes = [vp, C.POINTER(_Tensor), u32, i32, u32, f64, f64, f64, f64, vp, vp]
    i64, heads = C.c_int64, vp              # heads: the bytes of an edgc_heads
    L.edgc_embed_forward.restype = i32
    L.edgc_embed_forward.argtypes = [vp, i32, vp, u64, u32, u32, vp, i32, i64, u64, f32, vp, u64, vp]
    L.edgc_reserve_embed.restype = i32
    L.edgc_reserve_embed.argtypes = [vp, u32, u32, u32]
    L.edgc_embed_backward.restype = i32
    L.edgc_embed_backward.argtypes = [vp, i32, vp, i32, i64, u64, vp, u64, u32, u32, f32, vp, u64, i32, vp]
    L.edgc_qk_norm_forward.restype = i32
    L.edgc_qk_norm_forward.argtypes = [vp, i32, u64, u32, u32, u32, heads, heads, vp, vp, vp, i32, vp, u32, i32, f32, heads, heads, vp]
    L.edgc_reserve_qk_norm.restype = i32
    L.edgc_reserve_qk_norm.argtypes = [vp, u32, u32, u32, u32]
    L.edgc_qk_norm_backward.restype = i32
    L.edgc_qk_norm_backward.argtypes = [vp, i32, u64, u32, u32, u32, heads, heads, heads, heads, vp, vp, vp, i32, vp, u32, i32, f32, heads, heads,
                                        vp, vp, vp]
    _lib = L
    return L


class _DevicePeaks(C.Structure):
    _fields_ = [("copy_gbs", C.c_double), ("read_gbs", C.c_double), ("mfma_bf16_tflops", C.c_double),
                ("bytes", C.c_uint64), ("write_gbs", C.c_double)]


class _Tensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("grad_out", C.c_void_p), ("residual", C.c_void_p),
                ("Q", C.c_void_p), ("P", C.c_void_p), ("ld", C.c_uint64), ("ld_out", C.c_uint64),
                ("m", C.c_uint32), ("n", C.c_uint32), ("ldq", C.c_uint32), ("ldp", C.c_uint32),
                ("residual_is_zero", C.c_int32), ("deferred", C.c_uint32)]


class _FF(C.Structure):
    _fields_ = [("w_gate", C.c_void_p), ("w_up", C.c_void_p), ("w_down", C.c_void_p), ("ld_gate", C.c_uint64),
                ("ld_up", C.c_uint64), ("ld_down", C.c_uint64), ("hidden", C.c_uint32), ("ff", C.c_uint32),
                ("dtype", C.c_int32), ("act", C.c_int32)]


# An edgc_heads: address, elements from a token and from a head to the next.  (A ctypes structure takes ten times as long to build.)
_pack_heads = struct.Struct("@PQQ").pack


@dataclass
class Tensor:
    """One entry of a batch: torch CUDA tensors (``residual``, ``Q``, ``P`` may be None for a
    tensor that is sent as it stands; 1-D gradients are taken as one row).  Gradients have contiguous rows
    (of any row stride), ``grad`` and ``grad_out`` one type and shape, and rows and columns are below
    2^32 each: a longer flat gradient is given in parts."""
    grad: object
    grad_out: object
    residual: object = None
    Q: object = None
    P: object = None
    residual_is_zero: bool = False


class _RankCost(C.Structure):
    _fields_ = [("rank", C.c_uint32), ("_pad", C.c_uint32), ("t_compress", C.c_double),
                ("t_decompress", C.c_double), ("bytes_compressed", C.c_double)]


class _RankBounds(C.Structure):
    _fields_ = [("r_max", C.c_uint32), ("r_min", C.c_uint32), ("t_uncompressed", C.c_double)]


@dataclass
class RankCost:
    rank: int
    t_compress: float
    t_decompress: float
    bytes_compressed: float


@dataclass
class RankBounds:
    r_max: int
    r_min: int
    t_uncompressed: float
    t_com: List[float]


@dataclass
class EntropyResult:
    H_bits: float
    h_diff_nats: float
    lo: float
    hi: float
    n_sampled: int
    n_nonfinite: int
    status: int

    @staticmethod
    def from_buffer(buf) -> "EntropyResult":
        """Decode the raw result struct (e.g. a pinned uint8 tensor's bytes)."""
        r = _EntropyResult.from_buffer_copy(bytes(buf))
        return EntropyResult(r.H_bits, r.h_diff_nats, r.lo, r.hi, int(r.n_sampled),
                             int(r.n_nonfinite), int(r.status))


@dataclass
class RankParams:
    m: int
    n: int
    r_min: int
    r_max: int
    step_limit: int = 8
    allowed: Optional[Sequence[int]] = None
    eta: float = 0.0
    total_iters: int = 0
    min_warmup_frac: float = 0.10
    r_ref: int = 0


@dataclass
class RankState:
    have_ref: int = 0
    compressing: int = 0
    H_ref: float = 0.0
    r_prev: float = 0.0
    iters_seen: int = 0


@dataclass
class RankDecision:
    rank: int
    r_unclamped: float
    H_mean: float
    T_com: float


def select_rank(state: RankState, H_window: Sequence[float], iters_in_window: int,
                prm: RankParams) -> RankDecision:
    """edgc_select_rank: host-only; mutates ``state``."""
    L = load_library()
    H = (C.c_double * max(len(H_window), 1))(*[float(h) for h in H_window])
    p = _RankParams(prm.m, prm.n, prm.r_min, prm.r_max, prm.step_limit, None, 0, prm.eta,
                    prm.total_iters, prm.min_warmup_frac, prm.r_ref)
    keep = None
    if prm.allowed:
        keep = (C.c_uint32 * len(prm.allowed))(*prm.allowed)
        p.allowed = C.cast(keep, C.POINTER(C.c_uint32))
        p.n_allowed = len(prm.allowed)
    st = _RankState(state.have_ref, state.compressing, state.H_ref, state.r_prev, state.iters_seen)
    dec = _RankDecision()
    rc = L.edgc_select_rank(C.byref(st), C.cast(H, C.c_void_p), len(H_window), iters_in_window,
                            C.byref(p), C.byref(dec))
    if rc != OK:
        raise EdgcError(rc, "edgc_select_rank")
    state.have_ref, state.compressing = st.have_ref, st.compressing
    state.H_ref, state.r_prev, state.iters_seen = st.H_ref, st.r_prev, int(st.iters_seen)
    return RankDecision(int(dec.rank), dec.r_unclamped, dec.H_mean, dec.T_com)


def rank_bounds(costs: Sequence[RankCost], bytes_original: float, bandwidth: float,
                r_min_divisor: float = 4.0) -> RankBounds:
    """edgc_rank_bounds: host-only."""
    L = load_library()
    arr = (_RankCost * max(len(costs), 1))()
    for i, c in enumerate(costs):
        arr[i] = _RankCost(c.rank, 0, c.t_compress, c.t_decompress, c.bytes_compressed)
    out = _RankBounds()
    t = (C.c_double * max(len(costs), 1))()
    rc = L.edgc_rank_bounds(arr, len(costs), bytes_original, bandwidth, r_min_divisor, C.byref(out), t)
    if rc != OK:
        raise EdgcError(rc, "edgc_rank_bounds")
    return RankBounds(int(out.r_max), int(out.r_min), out.t_uncompressed, list(t)[:len(costs)])


def fit_eta(ranks: Sequence[int], t_com: Sequence[float]):
    """edgc_fit_eta: host-only.  Returns (eta, MAPE in percent)."""
    L = load_library()
    n = len(ranks)
    r = (C.c_uint32 * max(n, 1))(*[int(x) for x in ranks])
    t = (C.c_double * max(n, 1))(*[float(x) for x in t_com][:n])
    eta, mape = C.c_double(0), C.c_double(0)
    rc = L.edgc_fit_eta(r, t, n if len(t_com) == n else 0, C.byref(eta), C.byref(mape))
    if rc != OK:
        raise EdgcError(rc, "edgc_fit_eta")
    return eta.value, mape.value


def stage_ranks(r_stage1: int, t_microback: float, eta: float, r_min: int, r_max: int, n_stages: int,
                allowed: Optional[Sequence[int]] = None):
    """edgc_stage_ranks: host-only.  Returns (ranks per stage, predicted T_com per stage)."""
    L = load_library()
    ranks = (C.c_uint32 * max(n_stages, 1))()
    t = (C.c_double * max(n_stages, 1))()
    al = (C.c_uint32 * len(allowed))(*allowed) if allowed else None
    rc = L.edgc_stage_ranks(r_stage1, t_microback, eta, r_min, r_max, al, len(allowed) if allowed else 0,
                            n_stages, ranks, t)
    if rc != OK:
        raise EdgcError(rc, "edgc_stage_ranks")
    return [int(x) for x in ranks][:n_stages], list(t)[:n_stages]


def entropy_due(iter_in_window: int, period: int) -> bool:
    """edgc_entropy_due: host-only."""
    rc = load_library().edgc_entropy_due(iter_in_window, period)
    if rc < 0:
        raise EdgcError(rc, "edgc_entropy_due")
    return bool(rc)


def tensor_bypassed(m: int, n: int, r: int) -> bool:
    """edgc_tensor_bypassed: True when an m x n tensor is sent as it stands at rank r."""
    rc = load_library().edgc_tensor_bypassed(m, n, r)
    if rc < 0:
        raise EdgcError(rc, "edgc_tensor_bypassed")
    return bool(rc)


_torch = None           # the module, its two gradient types and its getter of a raw stream, from the first call that needs them
_codes: dict = {}
_raw_stream = None


def _load_torch():
    global _torch, _raw_stream
    import torch
    _codes.update({torch.float32: F32, torch.bfloat16: BF16})
    raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    _raw_stream = (lambda: raw(dev())) if raw and dev else None
    _torch = torch
    return torch


def _dtype_code(t) -> int:
    if _torch is None:
        _load_torch()
    code = _codes.get(t.dtype)
    if code is None:
        raise TypeError("gradient tensors must be float32 or bfloat16")
    return code


def _stream_handle(stream) -> int:
    """The stream's handle; without one that of torch's current stream, without the Stream object that
    torch.cuda.current_stream() builds (2.9 us of host time per call, of the 8 to 20 us that an entry point takes)."""
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch or _load_torch()
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream()
    return int(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return t.data_ptr() if t is not None else None


ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}


def _rows(name, t, dtype, shape) -> int:
    """Leading dimension of a matrix of that dtype and shape whose rows are contiguous."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    rows, cols = shape
    if t.shape != shape:
        raise ValueError(f"{name} must be of shape {tuple(shape)}")
    ld, step = t.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return ld if rows > 1 else cols


def _check_u32(*sizes) -> None:
    """Sizes that travel in 32 bits."""
    for n in sizes:
        if n >> 32:
            raise ValueError("tokens and widths must be 0 or more and below 2^32")


def _heads(name, t, dtype, shape) -> bytes:
    """The edgc_heads of queries or keys (tokens x heads x dim) of that dtype and shape, the dimensions of a head adjacent."""
    if t is None:
        raise ValueError(f"{name} is missing")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be of shape {tuple(shape)}")
    token, head, step = t.stride()
    if step != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have the dimensions of a head next to each other")
    return _pack_heads(t.data_ptr(), token, head)


def _integers(name, t, shape) -> int:
    """Bytes of an element of a contiguous vector of int32 or int64."""
    torch = _torch or _load_torch()
    if t.dtype is not torch.int64 and t.dtype is not torch.int32:
        raise TypeError(f"{name} must be int32 or int64")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous of shape {tuple(shape)}")
    return 8 if t.dtype is torch.int64 else 4


def _gradient_rows(t):
    """Rows, columns and leading dimension of a gradient, a matrix of contiguous rows or a contiguous vector (one row)."""
    shape, st = t.shape, t.stride()
    if len(shape) == 2:
        (m, n), (ld, step) = shape, st
    elif len(shape) == 1:
        m, n, ld, step = 1, shape[0], shape[0], st[0]
    else:
        raise ValueError("a gradient must be a vector or a matrix")
    if step != 1 and n > 1:
        raise ValueError("a gradient must have contiguous rows: the neighbours in a row of this one are not adjacent")
    if m >> 32 or n >> 32:
        raise ValueError("a gradient has fewer than 2^32 rows and columns: give a longer one in parts")
    return m, n, ld


class FeedForward:
    """The weights of a gated feed-forward block as the library takes them (edgc_ff): w_gate and w_up ff x hidden, w_down
    hidden x ff, as torch.nn.Linear keeps them; ``act``: "silu", "gelu" or "gelu_tanh".  Pointers and shapes are those the
    tensors had when it was built."""

    def __init__(self, w_gate, w_up, w_down, act: str = "silu"):
        if act not in ACTIVATIONS:
            raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
        if w_gate.dim() != 2:
            raise ValueError("w_gate must be ff x hidden")
        self.ff, self.hidden = (int(d) for d in w_gate.shape)
        _check_u32(self.ff, self.hidden)
        self.dtype, self.act = w_gate.dtype, act
        self.weights = (w_gate, w_up, w_down)
        lds = [_rows(n, w, self.dtype, s) for n, w, s in (("w_gate", w_gate, (self.ff, self.hidden)),
                                                          ("w_up", w_up, (self.ff, self.hidden)),
                                                          ("w_down", w_down, (self.hidden, self.ff)))]
        self.c = _FF(*[w.data_ptr() for w in self.weights], *lds, self.hidden, self.ff, _dtype_code(w_gate), ACTIVATIONS[act])


def _bad_dense(names, tensors, dtype, shape):
    """What is wrong with the first of the given tensors that is not contiguous, of that dtype and of that shape."""
    for name, t in zip(names, tensors):
        if t is None or (t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous()):
            continue
        raise (TypeError(f"{name} must be {dtype}") if t.dtype != dtype else
               ValueError(f"{name} must be contiguous of shape {tuple(shape)}"))


def _check_dense(names, tensors, dtype, shape) -> None:
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.shape != shape or not t.is_contiguous()):
            _bad_dense(names, tensors, dtype, shape)


def _devices(tensors) -> set:
    """Where the gradients of a list, and what is made of them, lie."""
    return {g.get_device() for t in tensors for g in (t.grad, t.grad_out) if g is not None}


class PreparedBatch:
    """The descriptor array of a list of :class:`Tensor`, built once.  The batched calls take it in
    place of the list; only the two per-call flags are written again (``residual_is_zero`` from the
    Tensor objects, ``deferred`` from the call).  Pointers, shapes and leading dimensions are those
    the tensors had when it was built: build a new one after any of them changes."""

    def __init__(self, tensors: Sequence[Tensor]):
        self.tensors = list(tensors)
        self.arr, self.code = Context._marshal(self.tensors)
        self.devices = _devices(self.tensors)

    def __len__(self):
        return len(self.tensors)

    def refresh(self, deferred: bool):
        d = 1 if deferred else 0
        for i, t in enumerate(self.tensors):
            a = self.arr[i]
            a.residual_is_zero = 1 if t.residual_is_zero else 0
            a.deferred = d
        return self.arr, self.code


class Context:
    """Owns an ``edgc_ctx``.  Methods take torch CUDA tensors (device memory only) and
    enqueue on ``stream`` (default: torch's current stream); nothing synchronises."""

    def __init__(self, device: int = 0, max_bins: int = 65536, max_rank: int = 128,
                 max_rows: int = 20480, max_cols: int = 20480):
        self._L = load_library()
        h = C.c_void_p()
        rc = self._L.edgc_create(C.byref(h), device, max_bins, max_rank, max_rows, max_cols)
        if rc != OK:
            raise EdgcError(rc, "edgc_create")
        self._h = h
        self.device = device

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._L.edgc_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int, what: str) -> None:
        if rc != OK:
            msg = self._L.edgc_last_error(self._h)
            raise EdgcError(rc, what, msg.decode() if msg else "")

    # -- per-kernel event timing ---------------------------------------------
    def profile_begin(self, max_launches: int = 4096) -> None:
        self._check(self._L.edgc_profile_begin(self._h, max_launches), "edgc_profile_begin")

    def profile_end(self) -> dict:
        """Stops the timing; returns {kernel: dict(launches, total_ms, bytes, flops)}."""
        cap = 64
        arr = (_KernelStat * cap)()
        n = C.c_uint32(0)
        self._check(self._L.edgc_profile_end(self._h, arr, cap, C.byref(n)), "edgc_profile_end")
        return {arr[i].kernel.decode(): dict(launches=int(arr[i].launches), total_ms=arr[i].total_ms,
                                             bytes=arr[i].bytes, flops=arr[i].flops,
                                             event_overhead_ms=arr[i].event_overhead_ms)
                for i in range(min(cap, n.value))}

    # -- entropy -----------------------------------------------------------
    def entropy_estimate_noalloc(self, grad, stride: int, chunk: int, seed: int, step: int, bins: int,
                                 out_pinned, value_range=None, counts_out=None, stream=None) -> None:
        """edgc_entropy_estimate_noalloc: the estimate on the library's file-scope scratch array
        (bins <= 65536); ``out_pinned`` as for :meth:`entropy_estimate_async`."""
        rng = None
        if value_range is not None:
            rng = (C.c_float * 2)(float(value_range[0]), float(value_range[1]))
        rc = self._L.edgc_entropy_estimate_noalloc(
            self._h, grad.data_ptr(), _dtype_code(grad), grad.numel(), stride, chunk, seed, step, bins,
            C.cast(rng, C.c_void_p) if rng is not None else None, out_pinned.data_ptr(),
            counts_out.data_ptr() if counts_out is not None else None, _stream_handle(stream))
        self._check(rc, "edgc_entropy_estimate_noalloc")

    def entropy_estimate_async(self, grad, stride: int, chunk: int, seed: int, step: int, bins: int,
                               out_pinned, value_range=None, counts_out=None, stream=None) -> None:
        """edgc_entropy_estimate, or edgc_entropy_estimate_batch when ``grad`` is a list of tensors
        (one estimate over the union of their samples).  ``out_pinned``: pinned uint8 CPU tensor
        of ENTROPY_RESULT_BYTES bytes, valid after the stream is synchronised."""
        rng = None
        if value_range is not None:
            rng = (C.c_float * 2)(float(value_range[0]), float(value_range[1]))
        if isinstance(grad, (list, tuple)):
            k = len(grad)
            ptrs = (C.c_void_p * max(k, 1))(*[g.data_ptr() for g in grad])
            sizes = (C.c_uint64 * max(k, 1))(*[g.numel() for g in grad])
            first = grad[0].dtype if k else None
            if any(g.dtype is not first for g in grad):
                for g in grad:
                    _dtype_code(g)
                raise TypeError("all buffers of one estimate must have one dtype")
            rc = self._L.edgc_entropy_estimate_batch(
                self._h, ptrs, sizes, k, _dtype_code(grad[0]) if k else F32, stride, chunk, seed, step, bins,
                C.cast(rng, C.c_void_p) if rng is not None else None, out_pinned.data_ptr(),
                counts_out.data_ptr() if counts_out is not None else None, _stream_handle(stream))
            self._check(rc, "edgc_entropy_estimate_batch")
            return
        rc = self._L.edgc_entropy_estimate(
            self._h, grad.data_ptr(), _dtype_code(grad), grad.numel(), stride, chunk, seed, step, bins,
            C.cast(rng, C.c_void_p) if rng is not None else None, out_pinned.data_ptr(),
            counts_out.data_ptr() if counts_out is not None else None, _stream_handle(stream))
        self._check(rc, "edgc_entropy_estimate")

    def entropy_estimate(self, grad, stride: int, chunk: int, seed: int, step: int, bins: int,
                         value_range=None, counts_out=None, stream=None) -> EntropyResult:
        """Blocking convenience wrapper: runs the estimate and synchronises the stream."""
        import torch
        out = torch.empty(ENTROPY_RESULT_BYTES, dtype=torch.uint8, pin_memory=True)
        self.entropy_estimate_async(grad, stride, chunk, seed, step, bins, out, value_range,
                                    counts_out, stream)
        (stream if stream is not None else torch.cuda.current_stream()).synchronize()
        return EntropyResult.from_buffer(out.numpy().tobytes())

    def sample_indices(self, n_elems: int, stride: int, chunk: int, seed: int, step: int,
                       idx_out=None, stream=None) -> int:
        """edgc_sample_indices.  Returns the sample size; fills ``idx_out`` (int64 CUDA tensor)."""
        n = C.c_uint64(0)
        rc = self._L.edgc_sample_indices(
            self._h, n_elems, stride, chunk, seed, step,
            idx_out.data_ptr() if idx_out is not None else None,
            idx_out.numel() if idx_out is not None else 0, C.byref(n), _stream_handle(stream))
        self._check(rc, "edgc_sample_indices")
        return int(n.value)

    # -- compressor --------------------------------------------------------
    def init_q(self, Q, col_begin: int, col_end: int, seed: int, stream=None) -> None:
        assert Q.dim() == 2 and Q.is_contiguous()
        rc = self._L.edgc_init_q(self._h, Q.data_ptr(), Q.shape[0], Q.shape[1], col_begin, col_end,
                                 seed, _stream_handle(stream))
        self._check(rc, "edgc_init_q")

    def compress(self, grad, residual, residual_is_zero: bool, Q, P, r: int, power_iters: int = 1,
                 stream=None) -> None:
        """edgc_compress.  grad (m, n) fp32/bf16 (row stride = grad.stride(0)); residual (m, n)
        fp32 contiguous; Q (n, ldq) and P (m, ldp) fp32 contiguous with ldq, ldp >= r."""
        m, n = grad.shape
        rc = self._L.edgc_compress(
            self._h, grad.data_ptr(), _dtype_code(grad), m, n, grad.stride(0), residual.data_ptr(),
            1 if residual_is_zero else 0, Q.data_ptr(), Q.shape[1], P.data_ptr(), P.shape[1], r,
            power_iters, _stream_handle(stream))
        self._check(rc, "edgc_compress")

    def decompress(self, P, Q, r: int, residual, grad_out, stream=None) -> None:
        """edgc_decompress.  residual (m, n) holds D on entry and E_new on return."""
        m, n = grad_out.shape
        rc = self._L.edgc_decompress(
            self._h, P.data_ptr(), P.shape[1], Q.data_ptr(), Q.shape[1], m, n, r, residual.data_ptr(),
            grad_out.data_ptr(), _dtype_code(grad_out), grad_out.stride(0), _stream_handle(stream))
        self._check(rc, "edgc_decompress")

    def measure_rank_costs(self, grad, residual, Q, P, grad_out, ranks: Sequence[int], reps: int = 5,
                           stream=None, deferred: bool = False) -> List[RankCost]:
        """edgc_measure_rank_costs: times compress and decompress at each rank on these buffers
        (all overwritten except grad); synchronises the stream.  ``deferred``: time the deferred
        form of the residual."""
        m, n = grad.shape
        rk = (C.c_uint32 * max(len(ranks), 1))(*[int(r) for r in ranks])
        out = (_RankCost * max(len(ranks), 1))()
        rc = self._L.edgc_measure_rank_costs(
            self._h, grad.data_ptr(), _dtype_code(grad), m, n, grad.stride(0), residual.data_ptr(),
            Q.data_ptr(), Q.shape[1], P.data_ptr(), P.shape[1], grad_out.data_ptr(), rk, len(ranks),
            reps, 1 if deferred else 0, out, _stream_handle(stream))
        self._check(rc, "edgc_measure_rank_costs")
        return [RankCost(int(c.rank), c.t_compress, c.t_decompress, c.bytes_compressed)
                for c in list(out)[:len(ranks)]]

    def measure_device_peaks(self, buf_a, buf_b, reps: int = 10, stream=None) -> dict:
        """edgc_measure_device_peaks: what a plain copy, a plain read and a bf16 MFMA loop reach on
        this device; buf_a is read, buf_b overwritten (two tensors of equal size in bytes);
        synchronises the stream."""
        nbytes = buf_a.numel() * buf_a.element_size()
        if nbytes != buf_b.numel() * buf_b.element_size():
            raise ValueError("the two buffers must have the same size in bytes")
        out = _DevicePeaks()
        rc = self._L.edgc_measure_device_peaks(self._h, buf_a.data_ptr(), buf_b.data_ptr(), nbytes, reps,
                                               C.byref(out), _stream_handle(stream))
        self._check(rc, "edgc_measure_device_peaks")
        return {"copy_gbs": out.copy_gbs, "read_gbs": out.read_gbs,
                "mfma_bf16_tflops": out.mfma_bf16_tflops, "bytes": int(out.bytes),
                "write_gbs": out.write_gbs}

    # -- batched calls -----------------------------------------------------
    def reserve_batch(self, shapes: Sequence[Sequence[int]]) -> None:
        """edgc_reserve_batch: position i of later batches holds at most shapes[i] = (rows, cols)."""
        n = len(shapes)
        rows = (C.c_uint32 * max(n, 1))(*[int(s[0]) for s in shapes])
        cols = (C.c_uint32 * max(n, 1))(*[int(s[1]) for s in shapes])
        self._check(self._L.edgc_reserve_batch(self._h, rows, cols, n), "edgc_reserve_batch")

    @staticmethod
    def _marshal(tensors, deferred: bool = False):
        if isinstance(tensors, PreparedBatch):
            return tensors.refresh(deferred)
        arr = (_Tensor * max(len(tensors), 1))()
        code, dtype, deferred = F32, None, 1 if deferred else 0
        for i, t in enumerate(tensors):
            grad, out, residual, Q, P = t.grad, t.grad_out, t.residual, t.Q, t.P
            g = out if grad is None else grad
            m, n, ld = _gradient_rows(g)
            if g.dtype is not dtype:
                code = _dtype_code(g)
                if dtype is not None:
                    raise TypeError("all gradients of a batch must have one dtype")
                dtype = g.dtype
            ld_out = 0 if out is None else ld
            if out is not None and out is not g:
                mo, no, ld_out = _gradient_rows(out)
                if m and n:                                         # (an empty one is the library's to refuse)
                    if out.dtype is not dtype:
                        raise TypeError("grad_out must be of its gradient's type")
                    if mo != m or no != n:
                        raise ValueError("grad_out must be of its gradient's shape")
            arr[i] = _Tensor(None if grad is None else grad.data_ptr(), None if out is None else out.data_ptr(),
                             None if residual is None else residual.data_ptr(), None if Q is None else Q.data_ptr(),
                             None if P is None else P.data_ptr(), 0 if grad is None else ld, ld_out, m, n,
                             0 if Q is None else Q.shape[1], 0 if P is None else P.shape[1], 1 if t.residual_is_zero else 0, deferred)
        return arr, code

    def compress_batch(self, tensors: Sequence[Tensor], r: int, power_iters: int = 1, stream=None,
                       deferred: bool = False) -> None:
        """edgc_compress_batch over a list of :class:`Tensor`; ``deferred``: the residual buffers
        hold D of the previous step and P, Q its factors (edgc_tensor.deferred of every entry)."""
        arr, code = self._marshal(tensors, deferred)
        rc = self._L.edgc_compress_batch(self._h, arr, len(tensors), code, r, power_iters,
                                         _stream_handle(stream))
        self._check(rc, "edgc_compress_batch")

    def compress_p_batch(self, tensors: Sequence[Tensor], r: int, stream=None, deferred: bool = False) -> None:
        """edgc_compress_p_batch: error-feedback add and P-pass; P is left un-orthonormalised."""
        arr, code = self._marshal(tensors, deferred)
        rc = self._L.edgc_compress_p_batch(self._h, arr, len(tensors), code, r, _stream_handle(stream))
        self._check(rc, "edgc_compress_p_batch")

    def compress_q_batch(self, tensors: Sequence[Tensor], r: int, stream=None) -> None:
        """edgc_compress_q_batch: orthonormalise P as it stands, then the Q-pass."""
        arr, code = self._marshal(tensors)
        rc = self._L.edgc_compress_q_batch(self._h, arr, len(tensors), code, r, _stream_handle(stream))
        self._check(rc, "edgc_compress_q_batch")

    def decompress_batch(self, tensors: Sequence[Tensor], r: int, stream=None, deferred: bool = False) -> None:
        """edgc_decompress_batch over a list of :class:`Tensor`; ``deferred``: only the
        reconstruction is written and the residual buffers keep D."""
        arr, code = self._marshal(tensors, deferred)
        rc = self._L.edgc_decompress_batch(self._h, arr, len(tensors), code, r, _stream_handle(stream))
        self._check(rc, "edgc_decompress_batch")

    def residual_materialize_batch(self, tensors: Sequence[Tensor], r: int, stream=None) -> None:
        """edgc_residual_materialize_batch: residual <- residual - round(P Q^T)."""
        arr, code = self._marshal(tensors)
        rc = self._L.edgc_residual_materialize_batch(self._h, arr, len(tensors), code, r,
                                                     _stream_handle(stream))
        self._check(rc, "edgc_residual_materialize_batch")

    # -- the block around the compressor --------------------------------------
    def _gradients(self, tensors):
        """Descriptors for the calls that read gradients alone: a prepared batch's as they are, without its per-call flags."""
        return (tensors.arr, tensors.code) if isinstance(tensors, PreparedBatch) else self._marshal(tensors)

    def grad_sumsq_batch(self, tensors: Sequence[Tensor], sumsq=None, accumulate: bool = False, stream=None) -> None:
        """edgc_grad_sumsq_batch: the sum of squares of the tensors' ``grad``, into ``sumsq`` (a float64 CUDA tensor of one
        element; None: the context's own place); ``accumulate`` adds to what is there."""
        if sumsq is not None and (sumsq.dtype != (_torch or _load_torch()).float64 or sumsq.numel() != 1):
            raise TypeError("sumsq must be one float64")
        arr, code = self._gradients(tensors)
        rc = self._L.edgc_grad_sumsq_batch(self._h, arr, len(tensors), code, 1 if accumulate else 0, _ptr(sumsq),
                                           _stream_handle(stream))
        self._check(rc, "edgc_grad_sumsq_batch")

    def clip_batch(self, tensors: Sequence[Tensor], max_norm: float, norm_coef=None, sumsq=None, stream=None) -> None:
        """edgc_clip_batch: ``grad_out`` = coefficient * ``grad``, by the sum of squares of the last
        :meth:`grad_sumsq_batch` (or ``sumsq``); ``norm_coef`` (float32 CUDA tensor of two) receives the norm and the
        coefficient."""
        torch = _torch or _load_torch()
        if sumsq is not None and (sumsq.dtype != torch.float64 or sumsq.numel() != 1):
            raise TypeError("sumsq must be one float64")
        if norm_coef is not None and (norm_coef.dtype != torch.float32 or norm_coef.numel() != 2 or not norm_coef.is_contiguous()):
            raise TypeError("norm_coef must be two float32")
        arr, code = self._gradients(tensors)
        rc = self._L.edgc_clip_batch(self._h, arr, len(tensors), code, float(max_norm), _ptr(sumsq), _ptr(norm_coef),
                                     _stream_handle(stream))
        self._check(rc, "edgc_clip_batch")

    def reserve_block_norm(self, tokens: int, hidden: int) -> None:
        """edgc_reserve_block_norm: scratch of :meth:`block_norm_backward` for up to that many tokens and hidden units, in place
        of an earlier reservation's limits.  Where its memory is not enough it is freed: capture graphs afterwards."""
        _check_u32(tokens, hidden)
        self._check(self._L.edgc_reserve_block_norm(self._h, tokens, hidden), "edgc_reserve_block_norm")

    @staticmethod
    def _norm_shapes(of, gate, rows_per_gate, names, dense, vectors, stats):
        """Tokens and hidden size of a pass whose tokens x hidden tensors are ``dense`` (and ``of``), whose vectors of hidden
        elements and of tokens statistics are the others; all as they have to be."""
        shape, dtype = of.shape, of.dtype
        if len(shape) != 2:
            raise ValueError("activations must be tokens x hidden")
        t, h = shape
        _check_dense(names[0], dense, dtype, shape)
        _check_dense(names[1], vectors, dtype, (h,))
        _check_dense(("rstd_post", "rstd_pre"), stats, _torch.float32, (t,))
        if gate is not None:
            if rows_per_gate < 1 or rows_per_gate >> 64:
                raise ValueError("rows_per_gate must be >= 1 with a gate, and below 2^64")
            _check_dense(("gate",), (gate,), dtype, (-(-t // rows_per_gate), h))
        return t, h

    def block_norm_forward(self, x, y, w_post, gate, w_pre, x_out, n_out, rstd_post=None, rstd_pre=None, scale: float = 1.0,
                           eps: float = 1e-6, rows_per_gate: int = 0, stream=None) -> None:
        """edgc_block_norm_forward: x_out = x + scale * gate * (norm(y) * w_post), n_out = norm(x_out) * w_pre; tokens x hidden.
        ``y`` None: the norm before a block alone; ``w_pre`` None: the norm after it alone."""
        code = _dtype_code(x)
        t, h = self._norm_shapes(x, gate, rows_per_gate, (("x", "y", "x_out", "n_out"), ("w_post", "w_pre")), (x, y, x_out, n_out),
                                 (w_post, w_pre), (rstd_post, rstd_pre))
        rc = self._L.edgc_block_norm_forward(self._h, code, t, h, x.data_ptr(), _ptr(y), _ptr(w_post), _ptr(gate), rows_per_gate,
                                             _ptr(w_pre), scale, eps, _ptr(x_out), _ptr(n_out), _ptr(rstd_post), _ptr(rstd_pre),
                                             _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_block_norm_forward")

    def block_norm_backward(self, dx_out, dn, x_out, y, w_post, gate, w_pre, rstd_post, rstd_pre, dx, dy, dw_post, dgate, dw_pre,
                            scale: float = 1.0, rows_per_gate: int = 0, stream=None) -> None:
        """edgc_block_norm_backward: the gradients of what :meth:`block_norm_forward` computed, from those of x_out and n_out."""
        code = _dtype_code(dx)
        t, h = self._norm_shapes(dx, gate, rows_per_gate, (("dx_out", "dn", "x_out", "y", "dx", "dy"), ("w_post", "w_pre", "dw_post", "dw_pre")),
                                 (dx_out, dn, x_out, y, dx, dy), (w_post, w_pre, dw_post, dw_pre), (rstd_post, rstd_pre))
        if gate is not None:
            _check_dense(("dgate",), (dgate,), dx.dtype, gate.shape)
        rc = self._L.edgc_block_norm_backward(self._h, code, t, h, _ptr(dx_out), _ptr(dn), _ptr(x_out), _ptr(y), _ptr(w_post),
                                              _ptr(gate), rows_per_gate, _ptr(w_pre), _ptr(rstd_post), _ptr(rstd_pre), scale,
                                              dx.data_ptr(), _ptr(dy), _ptr(dw_post), _ptr(dgate), _ptr(dw_pre), _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_block_norm_backward")

    def reserve_ff(self, dtype, tokens: int, hidden: int, ff: int, backward: bool = False) -> None:
        """edgc_reserve_ff: scratch of :meth:`ff_forward` (and :meth:`ff_backward`) for up to that many tokens of that
        width, in place of an earlier reservation (see :meth:`reserve_block_norm`); ``dtype``: torch.float32 or torch.bfloat16."""
        if _torch is None:
            _load_torch()
        if dtype not in _codes:
            raise TypeError("dtype must be float32 or bfloat16")
        _check_u32(tokens, hidden, ff)
        self._check(self._L.edgc_reserve_ff(self._h, _codes[dtype], tokens, hidden, ff, 1 if backward else 0), "edgc_reserve_ff")

    def ff_forward(self, ff: FeedForward, x, y, gate=None, up=None, stream=None) -> None:
        """edgc_ff_forward: y = (act(x w_gate^T) * (x w_up^T)) w_down^T; x, y tokens x hidden.  ``gate``, ``up`` (tokens x ff)
        keep the two projections for :meth:`ff_backward`."""
        t = x.shape[0]
        _check_u32(t)
        ldx, ldy = _rows("x", x, ff.dtype, (t, ff.hidden)), _rows("y", y, ff.dtype, (t, ff.hidden))
        ldk = 0
        if gate is not None and up is not None:
            ldk = _rows("gate", gate, ff.dtype, (t, ff.ff))
            if _rows("up", up, ff.dtype, (t, ff.ff)) != ldk:
                raise ValueError("gate and up must have one row stride")
        rc = self._L.edgc_ff_forward(self._h, C.byref(ff.c), x.data_ptr(), ldx, t, y.data_ptr(), ldy, _ptr(gate), _ptr(up), ldk,
                                     _stream_handle(stream))
        self._check(rc, "edgc_ff_forward")

    def ff_backward(self, ff: FeedForward, x, gate, up, dy, dx, dw_gate, dw_up, dw_down, accumulate: bool = False,
                    stream=None) -> None:
        """edgc_ff_backward: the gradients of x and of the three weights from dy, x and the kept projections; ``accumulate``
        adds the weights' gradients to what is there."""
        t, dt, th, tf = x.shape[0], ff.dtype, (x.shape[0], ff.hidden), (x.shape[0], ff.ff)
        _check_u32(t)
        ldk = _rows("gate", gate, dt, tf)
        if _rows("up", up, dt, tf) != ldk:
            raise ValueError("gate and up must have one row stride")
        rc = self._L.edgc_ff_backward(
            self._h, C.byref(ff.c), x.data_ptr(), _rows("x", x, dt, th), t, gate.data_ptr(), up.data_ptr(), ldk, dy.data_ptr(),
            _rows("dy", dy, dt, th), dx.data_ptr(), _rows("dx", dx, dt, th), dw_gate.data_ptr(),
            _rows("dw_gate", dw_gate, dt, (ff.ff, ff.hidden)), dw_up.data_ptr(), _rows("dw_up", dw_up, dt, (ff.ff, ff.hidden)),
            dw_down.data_ptr(), _rows("dw_down", dw_down, dt, (ff.hidden, ff.ff)), 1 if accumulate else 0, _stream_handle(stream))
        self._check(rc, "edgc_ff_backward")

    # -- before and after the stack of blocks --------------------------------------
    @staticmethod
    def _code_of(dtype) -> int:
        if _torch is None:
            _load_torch()
        if dtype not in _codes:
            raise TypeError("dtype must be float32 or bfloat16")
        return _codes[dtype]

    def reserve_orthogonalize(self, dtype, shapes: Sequence[Sequence[int]], steps: int = 5) -> None:
        """edgc_reserve_orthogonalize: scratch of :meth:`orthogonalize_batch` for lists of matrices none of which is larger than
        these, (rows, cols) each, in place of an earlier reservation (see :meth:`reserve_block_norm`)."""
        n, code = len(shapes), self._code_of(dtype)
        _check_u32(steps, *(d for s in shapes for d in s))
        rows = (C.c_uint32 * max(n, 1))(*[s[0] for s in shapes])
        cols = (C.c_uint32 * max(n, 1))(*[s[1] for s in shapes])
        self._check(self._L.edgc_reserve_orthogonalize(self._h, code, rows, cols, n, steps), "edgc_reserve_orthogonalize")

    def orthogonalize_batch(self, tensors: Sequence[Tensor], steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                            scales: Optional[Sequence[float]] = None, stream=None) -> None:
        """edgc_orthogonalize_batch: ``grad_out`` = scale * (``steps`` Newton-Schulz steps of ``grad`` / its norm), each matrix by
        itself; ``scales``: one per tensor."""
        arr, code = self._gradients(tensors)
        n = len(tensors)
        if not (tensors.devices if isinstance(tensors, PreparedBatch) else _devices(tensors)) <= {self.device}:
            raise ValueError(f"tensors must be on the context's device, cuda:{self.device}")
        if scales is not None and len(scales) != n:
            raise ValueError("scales must be one per tensor")
        _check_u32(steps)
        a, b, c = coefficients
        s = (C.c_float * max(n, 1))(*scales) if scales is not None else None
        rc = self._L.edgc_orthogonalize_batch(self._h, arr, n, code, steps, a, b, c, eps, s, _stream_handle(stream))
        self._check(rc, "edgc_orthogonalize_batch")

    def _on_device(self, *tensors) -> None:
        """Every given tensor lies on the context's GPU: another address would be one for its kernels to fault on."""
        device = self.device
        for t in tensors:
            if t is not None and t.get_device() != device:
                raise ValueError(f"tensors must be on the context's device, cuda:{self.device}")

    def embed_forward(self, table, ids, out, scale: float = 1.0, first_id: int = 0, stream=None) -> None:
        """edgc_embed_forward: out[t] = scale * table[ids[t] - first_id], zeros for an id that is not in the table; ``ids``: a contiguous
        vector of int32 or int64 (of a batch of sequences, ``ids.view(-1)``)."""
        if table.dim() != 2:
            raise ValueError("table must be vocab x hidden")
        (vocab, hidden), dtype = table.shape, table.dtype
        _check_u32(vocab, hidden)
        code, t = _dtype_code(table), ids.numel()
        bytes_ = _integers("ids", ids, (t,))
        ld, ldo = _rows("table", table, dtype, (vocab, hidden)), _rows("out", out, dtype, (t, hidden))
        self._on_device(table, ids, out)
        if first_id.bit_length() > 63:
            raise ValueError("first_id beyond 2^62")
        rc = self._L.edgc_embed_forward(self._h, code, table.data_ptr(), ld, vocab, hidden, ids.data_ptr(), bytes_, first_id, t, scale, out.data_ptr(),
                                        ldo, _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_embed_forward")

    def reserve_embed(self, tokens: int, vocab: int, hidden: int) -> None:
        """edgc_reserve_embed: scratch of :meth:`embed_backward` for up to that many tokens, rows and columns, in place of an earlier reservation (see
        :meth:`reserve_block_norm`)."""
        _check_u32(tokens, vocab, hidden)
        self._check(self._L.edgc_reserve_embed(self._h, tokens, vocab, hidden), "edgc_reserve_embed")

    def embed_backward(self, ids, dy, dtable, scale: float = 1.0, first_id: int = 0, accumulate: bool = False, stream=None) -> None:
        """edgc_embed_backward: dtable[v] = scale * the sum of dy[t] over ids[t] - first_id = v, zeros without a token; ``accumulate`` adds to what is
        there."""
        if dtable.dim() != 2:
            raise ValueError("dtable must be vocab x hidden")
        (vocab, hidden), dtype = dtable.shape, dtable.dtype
        _check_u32(vocab, hidden)
        code, t = _dtype_code(dtable), ids.numel()
        bytes_ = _integers("ids", ids, (t,))
        ldt, ldy = _rows("dtable", dtable, dtype, (vocab, hidden)), _rows("dy", dy, dtype, (t, hidden))
        self._on_device(dtable, ids, dy)
        if first_id.bit_length() > 63:
            raise ValueError("first_id beyond 2^62")
        rc = self._L.edgc_embed_backward(self._h, code, ids.data_ptr(), bytes_, first_id, t, dy.data_ptr(), ldy, vocab, hidden, scale,
                                         dtable.data_ptr(), ldt, 1 if accumulate else 0, _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_embed_backward")

    def _qk_args(self, q, k, w_q, w_k, positions, inv_freq):
        """What the two passes have in common, all as it has to be: shapes of queries and keys, type and sizes, positions and frequencies."""
        sq = q.shape
        if len(sq) != 3 or (k is not None and len(k.shape) != 3):
            raise ValueError("queries and keys must be tokens x heads x dim")
        t, hq, dim = sq
        hk = 0 if k is None else k.shape[1]
        if (hq | hk | dim) >> 32:
            _check_u32(hq, hk, dim)
        code, dtype = _dtype_code(q), q.dtype
        if w_q is None or (k is None) != (w_k is None):
            raise ValueError("queries need w_q, and keys w_k")
        _check_dense(("w_q", "w_k"), (w_q, w_k), dtype, (dim,))
        if inv_freq is None or not inv_freq.numel():
            return sq, (t, hk, dim), (self._h, code, t, hq, hk, dim), (None, 8, None, 0)
        if positions is None:
            raise ValueError("inv_freq needs positions")
        bytes_, n = _integers("positions", positions, (t,)), inv_freq.numel()
        _check_dense(("inv_freq",), (inv_freq,), _torch.float64, (n,))
        return sq, (t, hk, dim), (self._h, code, t, hq, hk, dim), (positions.data_ptr(), bytes_, inv_freq.data_ptr(), 2 * n)

    def qk_norm_forward(self, q, k, w_q, w_k, positions, inv_freq, q_out, k_out, eps: float = 1e-6, interleaved: bool = False, stream=None) -> None:
        """edgc_qk_norm_forward: every head of ``q`` and ``k`` (tokens x heads x dim, any strides of tokens and heads; ``k`` may be None) normed, times
        its weight, and the first 2 * len(inv_freq) dimensions rotated by positions * inv_freq (int32 or int64, and float64; None: none are)."""
        sq, sk, sizes, angle = self._qk_args(q, k, w_q, w_k, positions, inv_freq)
        dtype = q.dtype
        hq, hq_out, hk, hk_out = _heads("q", q, dtype, sq), _heads("q_out", q_out, dtype, sq), None, None
        if k is not None:
            hk, hk_out = _heads("k", k, dtype, sk), _heads("k_out", k_out, dtype, sk)
        elif k_out is not None:
            raise ValueError("k_out without keys")
        self._on_device(q, k, w_q, w_k, positions, inv_freq, q_out, k_out)
        rc = self._L.edgc_qk_norm_forward(*sizes, hq, hk, w_q.data_ptr(), _ptr(w_k), *angle, 1 if interleaved else 0, eps, hq_out, hk_out,
                                          _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_qk_norm_forward")

    def reserve_qk_norm(self, tokens: int, heads_q: int, heads_k: int, dim: int) -> None:
        """edgc_reserve_qk_norm: scratch of :meth:`qk_norm_backward` for up to these sizes, in place of an earlier reservation (see
        :meth:`reserve_block_norm`)."""
        _check_u32(tokens, heads_q, heads_k, dim)
        self._check(self._L.edgc_reserve_qk_norm(self._h, tokens, heads_q, heads_k, dim), "edgc_reserve_qk_norm")

    def qk_norm_backward(self, dq_out, dk_out, q, k, w_q, w_k, positions, inv_freq, dq, dk, dw_q, dw_k, eps: float = 1e-6, interleaved: bool = False,
                         stream=None) -> None:
        """edgc_qk_norm_backward: the gradients of what :meth:`qk_norm_forward` read, from those of what it wrote."""
        sq, sk, sizes, angle = self._qk_args(q, k, w_q, w_k, positions, inv_freq)
        dtype = q.dtype
        hq, hdy_q, hdx_q, hk, hdy_k, hdx_k = _heads("q", q, dtype, sq), _heads("dq_out", dq_out, dtype, sq), _heads("dq", dq, dtype, sq), None, None, None
        if k is not None:
            hk, hdy_k, hdx_k = _heads("k", k, dtype, sk), _heads("dk_out", dk_out, dtype, sk), _heads("dk", dk, dtype, sk)
        elif dk_out is not None or dk is not None:
            raise ValueError("dk_out or dk without keys")
        if dw_q is None or (k is None) != (dw_k is None):
            raise ValueError("queries need dw_q, and keys dw_k")
        _check_dense(("dw_q", "dw_k"), (dw_q, dw_k), dtype, (sq[2],))
        self._on_device(q, k, w_q, w_k, positions, inv_freq, dq_out, dk_out, dq, dk, dw_q, dw_k)
        rc = self._L.edgc_qk_norm_backward(*sizes, hdy_q, hdy_k, hq, hk, w_q.data_ptr(), _ptr(w_k), *angle, 1 if interleaved else 0, eps, hdx_q, hdx_k,
                                           dw_q.data_ptr(), _ptr(dw_k), _stream_handle(stream))
        if rc:
            self._check(rc, "edgc_qk_norm_backward")
