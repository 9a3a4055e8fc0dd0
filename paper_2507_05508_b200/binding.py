"""ctypes binding of libmlmc.so: argument marshalling only.

Every function has the name and the argument order of its C entry point in include/mlmc.h; torch
tensors are passed as raw device pointers and the current torch CUDA stream as the stream.  There is
no CPU path: if the CUDA library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmlmc.so")

MLMC_F32, MLMC_BF16 = 0, 1
MLMC_TOPK, MLMC_BITWISE, MLMC_RTN = 0, 1, 2
MLMC_OK = 0
MLMC_ERR_ARG, MLMC_ERR_SCHEDULE, MLMC_ERR_PROB, MLMC_ERR_CAPACITY = -1, -2, -3, -4
MLMC_ERR_NONFINITE, MLMC_ERR_TIMEOUT, MLMC_ERR_CUDA, MLMC_ERR_NOMEM, MLMC_ERR_INTERNAL = -5, -6, -7, -8, -9
MLMC_MAX_LEVELS = 32
MLMC_MAX_VOCAB, MLMC_MAX_TOP_LOGITS, MLMC_MAX_BEAMS, MLMC_MAX_BEAMS_OUT = 1 << 20, 1024, 32, 64

EXPORTS = ["mlmc_create", "mlmc_destroy", "mlmc_get_status", "mlmc_launch_count", "mlmc_read_u", "mlmc_read_listed_tiles",
           "mlmc_read_bracket_stats", "mlmc_read_sample_stats",
           "mlmc_kernel_count", "mlmc_kernel_name", "mlmc_timing_enable", "mlmc_timing_read",
           "mlmc_level_probs", "mlmc_compress_topk", "mlmc_compress_bitwise", "mlmc_aggregate",
           "mlmc_aggregate_topk_noalloc", "mlmc_compress_stopk", "mlmc_compress_floatbits", "mlmc_aggregate_floatbits",
           "mlmc_compress_rtn", "mlmc_aggregate_rtn", "mlmc_top_logits", "mlmc_distill", "mlmc_distill_grad",
           "mlmc_beam_select", "mlmc_beam_reorder"]


class MlmcError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where} returned status {code}")
        self.code = code


class mlmc_topk_msgs(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("val", C.c_void_p), ("count", C.c_void_p), ("level", C.c_void_p),
                ("p_sel", C.c_void_p), ("capacity", C.c_int64)]


class mlmc_bit_msgs(C.Structure):
    _fields_ = [("planes", C.c_void_p), ("gmax", C.c_void_p), ("level", C.c_void_p), ("p_sel", C.c_void_p),
                ("w_max", C.c_int32)]


class mlmc_float_msgs(C.Structure):
    _fields_ = [("expo", C.c_void_p), ("planes", C.c_void_p), ("level", C.c_void_p), ("p_sel", C.c_void_p),
                ("w_max", C.c_int32)]


class mlmc_rtn_msgs(C.Structure):
    _fields_ = [("val", C.c_void_p), ("c", C.c_void_p), ("level", C.c_void_p), ("p_sel", C.c_void_p),
                ("ldv", C.c_int64)]


class mlmc_logit_msgs(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("val", C.c_void_p), ("count", C.c_void_p), ("rest", C.c_void_p), ("k", C.c_int32)]


class mlmc_beams(C.Structure):
    _fields_ = [("token", C.c_void_p), ("parent", C.c_void_p), ("score", C.c_void_p), ("done", C.c_void_p)]


class mlmc_beam_state(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("beam_stride", C.c_int64), ("chunks", C.c_int64),
                ("chunk_stride", C.c_int64), ("chunk_bytes", C.c_int64)]


_lib = None


def lib() -> C.CDLL:
    """The CUDA library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2507_05508_b200.build` "
                                    "(or __graft_entry__.build()) first; there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int, C.c_int64, C.c_uint64
        L.mlmc_create.argtypes = [C.POINTER(vp), i32, i64, i32, i32]
        L.mlmc_destroy.argtypes = [vp]
        L.mlmc_get_status.argtypes = [vp, vp]
        L.mlmc_launch_count.argtypes = [vp]
        L.mlmc_launch_count.restype = i64
        L.mlmc_read_u.argtypes = [vp, u64, u64, i32, vp, vp]
        L.mlmc_read_listed_tiles.argtypes = [vp, i32, vp, vp, vp]
        L.mlmc_read_bracket_stats.argtypes = [vp, vp, vp]
        L.mlmc_read_sample_stats.argtypes = [vp, vp, vp]
        L.mlmc_level_probs.argtypes = [vp, vp, i32, i64, i32, i64, i32, vp, i32, vp, vp, vp, vp]
        L.mlmc_compress_topk.argtypes = [vp, vp, i32, i64, i32, i64, vp, i32, vp, u64, u64, vp, vp]
        L.mlmc_compress_bitwise.argtypes = [vp, vp, i32, i64, i32, i64, vp, i32, vp, u64, u64, vp, vp]
        L.mlmc_aggregate.argtypes = [vp, i32, vp, vp, i32, i32, i64, vp, vp]
        L.mlmc_aggregate_topk_noalloc.argtypes = [vp, i32, i64, vp, vp]
        L.mlmc_compress_stopk.argtypes = [vp, vp, i32, i64, i32, i64, i64, vp, u64, u64, vp, vp]
        L.mlmc_compress_floatbits.argtypes = [vp, vp, i32, i64, i32, i64, vp, i32, vp, u64, u64, vp, vp]
        L.mlmc_aggregate_floatbits.argtypes = [vp, vp, vp, i32, i32, i64, vp, vp]
        L.mlmc_compress_rtn.argtypes = [vp, vp, i32, i64, i32, i64, vp, i32, vp, u64, u64, vp, vp]
        L.mlmc_aggregate_rtn.argtypes = [vp, vp, i32, i64, vp, vp]
        f64 = C.c_double
        L.mlmc_top_logits.argtypes = [vp, vp, i32, i64, i64, i64, vp, f64, vp, vp]
        L.mlmc_distill.argtypes = [vp, vp, i32, i64, i64, i64, vp, f64, i32, vp, vp, vp, vp, i64, vp]
        L.mlmc_distill_grad.argtypes = [vp, vp, i32, i64, i64, i64, vp, f64, i32, vp, vp, vp, i64, vp]
        L.mlmc_beam_select.argtypes = [vp, vp, i64, i32, i32, f64, vp, vp, C.c_int32, i32, vp, vp]
        L.mlmc_beam_reorder.argtypes = [vp, vp, i32, i32, vp, i32, vp]
        L.mlmc_kernel_count.argtypes = []
        L.mlmc_kernel_name.argtypes = [i32]
        L.mlmc_timing_enable.argtypes = [vp, i32]
        L.mlmc_timing_read.argtypes = [vp, vp, vp, vp]
        for name in EXPORTS:
            if name not in ("mlmc_launch_count", "mlmc_kernel_name"):
                getattr(L, name).restype = i32
        L.mlmc_kernel_name.restype = C.c_char_p
        _lib = L
    return _lib


# The handle of the current stream without building a torch.cuda.Stream object (1.5 us a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


def _dtype_code(g: torch.Tensor) -> int:
    if g.dtype == torch.float32:
        return MLMC_F32
    if g.dtype == torch.bfloat16:
        return MLMC_BF16
    raise TypeError("gradients must be float32 or bfloat16")


def _check(rc: int, where: str) -> None:
    if rc != MLMC_OK:
        raise MlmcError(rc, where)


_host_arrays = {}     # (ctype, values) -> C array: a program hands over the same few schedules and probabilities step after step
_HOST_ARRAYS_MOST = 64
_HOST_ARRAY_LONGEST = 64      # (1000 numbers: 31 us to look up, 21 us to convert)


_PLAIN = {True: frozenset((float, np.float64)), False: frozenset((int, np.int64, np.int32))}


def _plain(ctype, values) -> bool:
    """Only numbers that the C array takes, and takes alike where they compare equal (1.0 and 1 do, and c_int64 refuses one)."""
    return type(values) in (list, tuple) and len(values) <= _HOST_ARRAY_LONGEST and \
        _PLAIN[ctype is C.c_double].issuperset(map(type, values))


def _host_array(ctype, values: Optional[Sequence]):
    """The values as a C array (read only for the library); one of plain numbers is kept for the next call with equal values."""
    if values is None:
        return None
    if not _plain(ctype, values):
        values = list(values)
        return (ctype * len(values))(*values)
    key = (ctype, tuple(values))
    a = _host_arrays.get(key)
    if a is None:
        if len(_host_arrays) >= _HOST_ARRAYS_MOST:
            _host_arrays.clear()
        a = _host_arrays[key] = (ctype * len(key[1]))(*key[1])
    return a


def mlmc_create(device: int, d_max: int, M_max: int, L_max: int) -> C.c_void_p:
    ctx = C.c_void_p()
    _check(lib().mlmc_create(C.byref(ctx), device, d_max, M_max, L_max), "mlmc_create")
    ctx.device = device
    return ctx


def mlmc_destroy(ctx) -> None:
    _check(lib().mlmc_destroy(ctx), "mlmc_destroy")


def mlmc_get_status(ctx) -> int:
    return int(lib().mlmc_get_status(ctx, _stream()))


def mlmc_launch_count(ctx) -> int:
    return int(lib().mlmc_launch_count(ctx))


def mlmc_kernel_count() -> int:
    return int(lib().mlmc_kernel_count())


def mlmc_kernel_name(i: int) -> str:
    return lib().mlmc_kernel_name(i).decode()


def mlmc_timing_enable(ctx, on: bool) -> None:
    _check(lib().mlmc_timing_enable(ctx, 1 if on else 0), "mlmc_timing_enable")


def mlmc_timing_read(ctx):
    """{kernel name: (total ms, launches)} recorded since the previous read (synchronises the stream)."""
    n = mlmc_kernel_count()
    ms, cnt = (C.c_double * n)(), (C.c_int64 * n)()
    _check(lib().mlmc_timing_read(ctx, ms, cnt, _stream()), "mlmc_timing_read")
    return {mlmc_kernel_name(i): (ms[i], cnt[i]) for i in range(n) if cnt[i]}


def mlmc_read_u(ctx, seed: int, step: int, M: int):
    buf = (C.c_double * M)()
    _check(lib().mlmc_read_u(ctx, seed, step, M, buf, _stream()), "mlmc_read_u")
    return list(buf)


def mlmc_read_listed_tiles(ctx, M: int):
    """(tiles read per worker by the last Top-k emission, tiles per row)."""
    buf = (C.c_uint32 * M)()
    tiles = C.c_int64(0)
    _check(lib().mlmc_read_listed_tiles(ctx, M, buf, C.byref(tiles), _stream()), "mlmc_read_listed_tiles")
    return list(buf), int(tiles.value)


def mlmc_read_bracket_stats(ctx):
    """(workers whose brackets held, workers with a missed bracket, workers without a stored bin), cumulative."""
    buf = (C.c_uint64 * 3)()
    _check(lib().mlmc_read_bracket_stats(ctx, buf, _stream()), "mlmc_read_bracket_stats")
    return tuple(int(x) for x in buf)


def mlmc_read_sample_stats(ctx):
    """Sampled brackets: (workers whose brackets held, workers with one that missed, workers of calls left out), cumulative."""
    buf = (C.c_uint64 * 3)()
    _check(lib().mlmc_read_sample_stats(ctx, buf, _stream()), "mlmc_read_sample_stats")
    return tuple(int(x) for x in buf)


def _g_args(g: torch.Tensor):
    assert g.is_cuda and g.dim() == 2 and g.stride(1) == 1
    return g.data_ptr(), _dtype_code(g), g.shape[1], g.shape[0], g.stride(0)


def mlmc_level_probs(ctx, g: torch.Tensor, kind: int, sched: Sequence[int], p: Optional[Sequence[float]],
                     p_out: torch.Tensor, delta_out: Optional[torch.Tensor]) -> None:
    ptr, dt, d, M, ld = _g_args(g)
    sch = _host_array(C.c_int64, sched)
    ph = _host_array(C.c_double, p)
    L = len(sched) + (1 if kind == MLMC_RTN else 0)      # the RTN schedule lists the widths below the identity level
    _check(lib().mlmc_level_probs(ctx, ptr, dt, d, M, ld, kind, sch, L, ph, p_out.data_ptr(),
                                  None if delta_out is None else delta_out.data_ptr(), _stream()), "mlmc_level_probs")


def mlmc_compress_topk(ctx, g: torch.Tensor, k: Sequence[int], p: Optional[Sequence[float]], seed: int, step: int,
                       out: "TopkBuffers") -> None:
    ptr, dt, d, M, ld = _g_args(g)
    kh = _host_array(C.c_int64, k)
    ph = _host_array(C.c_double, p)
    _check(lib().mlmc_compress_topk(ctx, ptr, dt, d, M, ld, kh, len(k), ph, seed, step, C.byref(out.struct),
                                    _stream()), "mlmc_compress_topk")


def mlmc_compress_bitwise(ctx, g: torch.Tensor, b: Sequence[int], p: Optional[Sequence[float]], seed: int, step: int,
                          out: "BitBuffers") -> None:
    ptr, dt, d, M, ld = _g_args(g)
    bh = _host_array(C.c_int32, b)
    ph = _host_array(C.c_double, p)
    _check(lib().mlmc_compress_bitwise(ctx, ptr, dt, d, M, ld, bh, len(b), ph, seed, step, C.byref(out.struct),
                                       _stream()), "mlmc_compress_bitwise")


def mlmc_aggregate(ctx, kind: int, msgs, b: Optional[Sequence[int]], M: int, d: int, out: torch.Tensor) -> None:
    assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.numel() >= d
    bh = _host_array(C.c_int32, b)
    _check(lib().mlmc_aggregate(ctx, kind, C.byref(msgs.struct), bh, 0 if b is None else len(b), M, d,
                                out.data_ptr(), _stream()), "mlmc_aggregate")


def mlmc_aggregate_topk_noalloc(msgs: "TopkBuffers", M: int, d: int, out: torch.Tensor) -> None:
    """Top-k server average that needs no context and allocates nothing (fixed built-in scratch; see mlmc.h)."""
    assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.numel() >= d
    _check(lib().mlmc_aggregate_topk_noalloc(C.byref(msgs.struct), M, d, out.data_ptr(), _stream()),
           "mlmc_aggregate_topk_noalloc")


def mlmc_compress_stopk(ctx, g: torch.Tensor, s: int, p: Optional[Sequence[float]], seed: int, step: int,
                        out: "TopkBuffers") -> None:
    ptr, dt, d, M, ld = _g_args(g)
    ph = None if p is None else _host_array(C.c_double, p) if _plain(C.c_double, p) else \
        (C.c_double * len(p)).from_buffer_copy(memoryview(_as_f64(p)))
    _check(lib().mlmc_compress_stopk(ctx, ptr, dt, d, M, ld, s, ph, seed, step, C.byref(out.struct), _stream()),
           "mlmc_compress_stopk")


def _as_f64(p):
    import numpy as np
    return np.ascontiguousarray(p, dtype=np.float64)


def mlmc_compress_floatbits(ctx, g: torch.Tensor, mb: Sequence[int], p: Optional[Sequence[float]], seed: int, step: int,
                            out: "FloatBuffers") -> None:
    ptr, dt, d, M, ld = _g_args(g)
    mh = _host_array(C.c_int32, mb)
    ph = _host_array(C.c_double, p)
    _check(lib().mlmc_compress_floatbits(ctx, ptr, dt, d, M, ld, mh, len(mb), ph, seed, step, C.byref(out.struct),
                                         _stream()), "mlmc_compress_floatbits")


def mlmc_aggregate_floatbits(ctx, msgs: "FloatBuffers", mb: Sequence[int], M: int, d: int, out: torch.Tensor) -> None:
    assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.numel() >= d
    mh = _host_array(C.c_int32, mb)
    _check(lib().mlmc_aggregate_floatbits(ctx, C.byref(msgs.struct), mh, len(mb), M, d, out.data_ptr(), _stream()),
           "mlmc_aggregate_floatbits")


def mlmc_compress_rtn(ctx, g: torch.Tensor, r: Sequence[int], p: Optional[Sequence[float]], seed: int, step: int,
                      out: "RtnBuffers") -> None:
    """r: the L - 1 round-to-nearest widths; level L - 1 is the identity."""
    ptr, dt, d, M, ld = _g_args(g)
    rh = _host_array(C.c_int32, r) if len(r) else None
    ph = _host_array(C.c_double, p)
    _check(lib().mlmc_compress_rtn(ctx, ptr, dt, d, M, ld, rh, len(r) + 1, ph, seed, step, C.byref(out.struct),
                                   _stream()), "mlmc_compress_rtn")


def mlmc_aggregate_rtn(ctx, msgs: "RtnBuffers", M: int, d: int, out: torch.Tensor) -> None:
    assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.numel() >= d
    _check(lib().mlmc_aggregate_rtn(ctx, C.byref(msgs.struct), M, d, out.data_ptr(), _stream()), "mlmc_aggregate_rtn")


# ---- what a model answers: top logits, distillation, beam search ----
def _rows(x: torch.Tensor):
    """Pointer, dtype code, V, N, ld of a [N, V] tensor of logits."""
    if not x.is_cuda or x.dim() != 2 or (x.shape[1] != 1 and x.stride(1) != 1):
        raise ValueError("logits are a [N, V] tensor on the GPU whose rows are contiguous")
    n, v = x.shape
    return x.data_ptr(), _dtype_code(x), v, n, x.stride(0) if n > 1 else v


def _vector(x: Optional[torch.Tensor], dtype, numel: int, device, what: str):
    """Pointer of a contiguous tensor of that type and size on that device; None for None."""
    if x is None:
        return None
    if x.dtype != dtype or x.numel() != numel or x.device != device or not x.is_contiguous():
        raise ValueError(f"{what} is a contiguous {dtype} tensor of {numel} elements on {device}")
    return x.data_ptr()


def _stream_of(ctx, device) -> int:
    """The current stream of the tensors' GPU, which has to be the context's: a kernel on another one cannot reach them."""
    if getattr(ctx, "device", device.index) != device.index:
        raise ValueError(f"the tensors are on {device}, the context is of GPU {ctx.device}")
    return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device.index)


def _messages(msgs: "LogitBuffers", n: int, device):
    if msgs.N != n or msgs.idx.device != device:
        raise ValueError(f"messages of {n} rows on {device} are needed, these are of {msgs.N} on {msgs.idx.device}")
    return msgs.ref


def mlmc_top_logits(ctx, logits: torch.Tensor, skip: Optional[torch.Tensor], T: float, out: "LogitBuffers") -> None:
    """The message of every row: its out.k largest logits, their indices, and the mass of the others; rows with skip != 0 have none."""
    ptr, dt, v, n, ld = _rows(logits)
    dev = logits.device
    _check(lib().mlmc_top_logits(ctx, ptr, dt, v, n, ld, _vector(skip, torch.uint8, n, dev, "skip"), T, _messages(out, n, dev),
                                 _stream_of(ctx, dev)), "mlmc_top_logits")


def _grad_rows(logits: torch.Tensor, grad: torch.Tensor):
    ptr, _, _, _, ld = _rows(grad)
    if grad.shape != logits.shape or grad.dtype != logits.dtype or grad.device != logits.device:
        raise ValueError("the gradient has the shape, the type and the device of the logits")
    return ptr, ld


def _loss_buffers(out: "DistillBuffers", n: int, device):
    if out.N != n or out.loss.device != device:
        raise ValueError(f"buffers of {n} rows on {device} are needed, these are of {out.N} on {out.loss.device}")


def mlmc_distill(ctx, logits: torch.Tensor, msgs: "LogitBuffers", T: float, rest: bool, weight: Optional[torch.Tensor],
                 out: "DistillBuffers", grad: Optional[torch.Tensor]) -> None:
    """out.loss[n] = T^2 KL(teacher || student) of every row, out.stat for mlmc_distill_grad; with grad also weight[n] dloss[n]/dlogits."""
    ptr, dt, v, n, ld = _rows(logits)
    dev = logits.device
    _loss_buffers(out, n, dev)
    gp, ldg = (None, v) if grad is None else _grad_rows(logits, grad)
    _check(lib().mlmc_distill(ctx, ptr, dt, v, n, ld, _messages(msgs, n, dev), T, 1 if rest else 0,
                              _vector(weight, torch.float32, n, dev, "weight"), out.loss_ptr, out.stat_ptr, gp, ldg,
                              _stream_of(ctx, dev)), "mlmc_distill")


def mlmc_distill_grad(ctx, logits: torch.Tensor, msgs: "LogitBuffers", T: float, rest: bool, weight: Optional[torch.Tensor],
                      out: "DistillBuffers", grad: torch.Tensor) -> None:
    """weight[n] dloss[n]/dlogits from the out.stat of mlmc_distill with the same logits, messages, T and rest."""
    ptr, dt, v, n, ld = _rows(logits)
    dev = logits.device
    _loss_buffers(out, n, dev)
    gp, ldg = _grad_rows(logits, grad)
    _check(lib().mlmc_distill_grad(ctx, ptr, dt, v, n, ld, _messages(msgs, n, dev), T, 1 if rest else 0,
                                   _vector(weight, torch.float32, n, dev, "weight"), out.stat_ptr, gp, ldg, _stream_of(ctx, dev)),
           "mlmc_distill_grad")


def mlmc_beam_select(ctx, rows: "LogitBuffers", V: int, W: int, T: float, score: torch.Tensor, done: Optional[torch.Tensor], eos: int,
                     out: "BeamBuffers") -> None:
    """The out.K best continuations of every sentence from the messages of its W beams' logits."""
    n, dev = out.B * W, rows.idx.device
    if out.token.device != dev:
        raise ValueError("the beams are on another device than the messages")
    _check(lib().mlmc_beam_select(ctx, _messages(rows, n, dev), V, out.B, W, T, _vector(score, torch.float32, n, dev, "score"),
                                  _vector(done, torch.uint8, n, dev, "done"), eos, out.K,
                                  out.ref if done is not None else out.ref_endless, _stream_of(ctx, dev)), "mlmc_beam_select")


def mlmc_beam_reorder(ctx, parent: torch.Tensor, states: "BeamStates") -> None:
    """Beam w of every sentence takes the states of beam parent[.., w]."""
    if parent.device != states.device or parent.numel() != states.beams or parent.dtype != torch.int32 or not parent.is_contiguous():
        raise ValueError(f"parent is a contiguous int32 tensor of {states.beams} elements on {states.device}")
    _check(lib().mlmc_beam_reorder(ctx, parent.data_ptr(), states.beams // states.W, states.W, states.array, states.n,
                                   _stream_of(ctx, states.device)), "mlmc_beam_reorder")


class LogitBuffers:
    """Caller-owned device buffers of the messages of N rows of logits."""

    def __init__(self, N: int, k: int, device: str = "cuda"):
        self._take(torch.empty((N, k), dtype=torch.int32, device=device),      # uint32 payload
                   torch.empty((N, k), dtype=torch.float32, device=device),
                   torch.zeros(N, dtype=torch.int32, device=device),
                   torch.full((N,), -float("inf"), dtype=torch.float32, device=device))

    @classmethod
    def of(cls, idx: torch.Tensor, val: torch.Tensor, count: torch.Tensor, rest: Optional[torch.Tensor]) -> "LogitBuffers":
        """Messages in buffers that exist already; rest may be None where only renormalised probabilities are used."""
        if not idx.is_cuda or idx.dim() != 2:
            raise ValueError("idx is a [N, k] tensor on the GPU")
        n, k = idx.shape
        dev = idx.device
        _vector(idx, torch.int32, n * k, dev, "idx")
        _vector(val, torch.float32, n * k, dev, "val")
        _vector(count, torch.int32, n, dev, "count")
        _vector(rest, torch.float32, n, dev, "rest")
        self = cls.__new__(cls)
        self._take(idx, val, count, rest)
        return self

    def _take(self, idx, val, count, rest):
        self.N, self.k = idx.shape
        self.idx, self.val, self.count, self.rest = idx, val, count, rest
        self.struct = mlmc_logit_msgs(idx.data_ptr(), val.data_ptr(), count.data_ptr(), None if rest is None else rest.data_ptr(), self.k)
        self.ref = C.byref(self.struct)


class DistillBuffers:
    """Caller-owned device buffers of a distillation loss: the loss of every row, and what its gradient needs later."""

    def __init__(self, N: int, device: str = "cuda"):
        self.N = N
        self.loss = torch.zeros(N, dtype=torch.float32, device=device)
        self.stat = torch.zeros((N, 8), dtype=torch.float32, device=device)
        self.loss_ptr, self.stat_ptr = self.loss.data_ptr(), self.stat.data_ptr()


class BeamBuffers:
    """Caller-owned device buffers of the beams that a step goes on with: B sentences, K places each."""

    def __init__(self, B: int, K: int, device: str = "cuda"):
        self.B, self.K = B, K
        self.token = torch.zeros((B, K), dtype=torch.int32, device=device)
        self.parent = torch.zeros((B, K), dtype=torch.int32, device=device)
        self.score = torch.full((B, K), -float("inf"), dtype=torch.float32, device=device)
        self.done = torch.zeros((B, K), dtype=torch.uint8, device=device)
        self.struct = mlmc_beams(self.token.data_ptr(), self.parent.data_ptr(), self.score.data_ptr(), self.done.data_ptr())
        self.endless = mlmc_beams(self.struct.token, self.struct.parent, self.struct.score, None)      # no token ends a beam
        self.ref, self.ref_endless = C.byref(self.struct), C.byref(self.endless)


_MOST_PIECES = 1 << 22


def _meet(entries, beams: int) -> bool:
    """Whether a state's destination shares bytes with another state (of views between one another up to _MOST_PIECES pieces are looked at)."""
    spans = []
    for e in entries:
        length = (beams - 1) * e.beam_stride + (e.chunks - 1) * e.chunk_stride + e.chunk_bytes
        spans.append((e.dst, length, True, e))
        if e.src != e.dst:
            spans.append((e.src, length, False, e))
    spans.sort(key=lambda x: x[0])
    written = anything = -1          # ends of what came before
    for first, length, dst, _ in spans:
        if first < (anything if dst else written):
            break
        anything = max(anything, first + length)
        if dst:
            written = max(written, first + length)
    else:
        return False
    if sum(beams * e.chunks for _, _, _, e in spans) > _MOST_PIECES:
        return False
    starts = [(first + np.arange(beams, dtype=np.int64)[:, None] * e.beam_stride + np.arange(e.chunks, dtype=np.int64) * e.chunk_stride).ravel()
              for first, _, _, e in spans]
    first = np.concatenate(starts)
    end = first + np.repeat([e.chunk_bytes for _, _, _, e in spans], [len(x) for x in starts])
    dst = np.repeat([d for _, _, d, _ in spans], [len(x) for x in starts])
    order = np.argsort(first, kind="stable")
    first, end, dst = first[order], end[order], dst[order]
    anything, written = np.maximum.accumulate(end), np.maximum.accumulate(np.where(dst, end, -1))
    return bool((first[1:] < np.where(dst[1:], anything[:-1], written[:-1])).any())


class BeamStates:
    """States of B * W beams: (source, destination) tensors [B * W, ...], or one tensor that is reordered in place.

    Behind the first dimension a state may be strided in one place (a cache [B * W, heads, room, size] cut to the tokens so far);
    source and destination have the same shape and strides, and no destination shares memory with another state.  The tensors are kept; their shapes and memory are looked up here and not
    again, which takes some 10 us of the host for each.  For caches that grow, `tokens` is the dimension along which they do (2 above):
    `first(n)` makes the next call move the first n tokens of it."""

    def __init__(self, states, W: int, tokens: Optional[int] = None):
        self.W, self.kept, entries, token_bytes = W, [], [], []
        self.device, self.beams, self.room = None, 0, None
        for pair in states:
            src, dst = pair if isinstance(pair, (tuple, list)) else (pair, pair)
            if not src.is_cuda or src.device != dst.device or src.dtype != dst.dtype or src.shape != dst.shape or src.dim() < 1:
                raise ValueError("source and destination are tensors of one shape, type and GPU")
            if self.device is None:
                self.device, self.beams = src.device, src.shape[0]
            if src.device != self.device or src.shape[0] != self.beams or self.beams % W:
                raise ValueError("every state has B * W beams in its first dimension, all on one GPU")
            if tokens is not None:
                if not 1 <= tokens < src.dim():
                    raise ValueError("tokens is a dimension behind the first one")
                self.room = src.shape[tokens] if self.room is None else min(self.room, src.shape[tokens])
            if src.numel() == 0:
                continue
            size = src.element_size()
            if any(src.stride(i) != dst.stride(i) for i in range(src.dim()) if src.shape[i] > 1):
                raise ValueError("source and destination have the same strides")
            dims = [i for i in range(1, src.dim()) if src.shape[i] > 1]
            chunk = size
            while dims and (tokens is None or dims[-1] > tokens) and src.stride(dims[-1]) * size == chunk:      # the contiguous piece at the end
                chunk *= src.shape[dims.pop()]
            if tokens is not None:
                token_bytes.append(chunk)
                if dims and dims[-1] == tokens and src.stride(tokens) * size == chunk:
                    chunk *= src.shape[dims.pop()]
                if dims and dims[-1] >= tokens:
                    raise ValueError("a state's tokens lie one behind the other")
            chunks, stride = 1, 0
            if dims:
                stride = src.stride(dims[-1]) * size
                chunks = src.shape[dims.pop()]
            while dims and src.stride(dims[-1]) * size == chunks * stride:
                chunks *= src.shape[dims.pop()]
            if dims:
                raise ValueError("a state may be strided in one place behind its first dimension")
            entries.append(mlmc_beam_state(src.data_ptr(), dst.data_ptr(), src.stride(0) * size if self.beams > 1 else 0, chunks, stride, chunk))
            self.kept.append((src, dst))
        if self.device is None:
            raise ValueError("there are no states")
        if _meet(entries, self.beams):
            raise ValueError("the destination of a state shares memory with another state")
        self.n = len(entries)
        self.array = (mlmc_beam_state * max(1, self.n))(*entries)
        self.token_bytes = np.array(token_bytes, dtype=np.int64)
        words = np.frombuffer(self.array, dtype=np.int64).reshape(-1, C.sizeof(mlmc_beam_state) // 8)
        self.chunk_bytes = words[:self.n, mlmc_beam_state.chunk_bytes.offset // 8]

    def first(self, n: int) -> "BeamStates":
        """The same states, of which the next calls move the first n tokens."""
        if self.room is None or not 0 <= n <= self.room:
            raise ValueError(f"0 to {self.room} tokens can be moved, not {n}" if self.room is not None else "these states have no dimension of tokens")
        np.multiply(self.token_bytes, n, out=self.chunk_bytes)
        return self


class FloatBuffers:
    """Caller-owned device buffers of a floating-point message batch."""

    def __init__(self, M: int, d: int, w_max: int, device: str = "cuda"):
        self.M, self.d, self.w_max = M, d, w_max
        self.words = (d + 31) // 32
        self.expo = torch.zeros((M, self.words * 32), dtype=torch.uint8, device=device)
        self.planes = torch.zeros((M, 1 + w_max, self.words), dtype=torch.int32, device=device)  # uint32 payload
        self.level = torch.full((M,), -1, dtype=torch.int32, device=device)
        self.p_sel = torch.zeros(M, dtype=torch.float64, device=device)
        self.struct = mlmc_float_msgs(self.expo.data_ptr(), self.planes.data_ptr(), self.level.data_ptr(),
                                      self.p_sel.data_ptr(), w_max)


class RtnBuffers:
    """Caller-owned device buffers of a dense MLMC-RTN message batch (rows padded to 16 bytes)."""

    def __init__(self, M: int, d: int, device: str = "cuda"):
        self.M, self.d = M, d
        self.ldv = (d + 3) // 4 * 4
        self.val = torch.zeros((M, self.ldv), dtype=torch.float32, device=device)
        self.c = torch.zeros(M, dtype=torch.float32, device=device)
        self.level = torch.full((M,), -1, dtype=torch.int32, device=device)
        self.p_sel = torch.zeros(M, dtype=torch.float64, device=device)
        self.struct = mlmc_rtn_msgs(self.val.data_ptr(), self.c.data_ptr(), self.level.data_ptr(),
                                    self.p_sel.data_ptr(), self.ldv)


class TopkBuffers:
    """Caller-owned device buffers of a Top-k message batch (torch only provides the memory)."""

    def __init__(self, M: int, capacity: int, device: str = "cuda"):
        self.M, self.capacity = M, capacity
        self.idx = torch.empty((M, max(capacity, 1)), dtype=torch.int32, device=device)   # uint32 payload
        self.val = torch.empty((M, max(capacity, 1)), dtype=torch.float32, device=device)
        self.count = torch.zeros(M, dtype=torch.int64, device=device)
        self.level = torch.full((M,), -1, dtype=torch.int32, device=device)
        self.p_sel = torch.zeros(M, dtype=torch.float64, device=device)
        self.struct = mlmc_topk_msgs(self.idx.data_ptr(), self.val.data_ptr(), self.count.data_ptr(),
                                     self.level.data_ptr(), self.p_sel.data_ptr(), capacity)


class BitBuffers:
    """Caller-owned device buffers of a bit-plane message batch."""

    def __init__(self, M: int, d: int, w_max: int, device: str = "cuda"):
        self.M, self.d, self.w_max = M, d, w_max
        self.words = (d + 31) // 32
        self.planes = torch.zeros((M, 1 + w_max, self.words), dtype=torch.int32, device=device)  # uint32 payload
        self.gmax = torch.zeros(M, dtype=torch.float32, device=device)
        self.level = torch.full((M,), -1, dtype=torch.int32, device=device)
        self.p_sel = torch.zeros(M, dtype=torch.float64, device=device)
        self.struct = mlmc_bit_msgs(self.planes.data_ptr(), self.gmax.data_ptr(), self.level.data_ptr(),
                                    self.p_sel.data_ptr(), w_max)
