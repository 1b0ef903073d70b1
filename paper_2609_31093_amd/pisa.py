"""Thin ctypes binding of libpisa (the C ABI declared in include/pisa.h).

Each ``pisa_*`` function here has the name and argument order of its C
counterpart; tensors are passed as device pointers and the stream defaults to
torch's current stream.  Every step of the computation runs in the HIP
library: this module only marshals arguments, allocates outputs with torch and
turns negative status codes into :class:`PisaError`.  It raises at import time
if the library has not been built (there is no fallback path).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpisa.so")

PISA_DTYPE_F32 = 0
PISA_DTYPE_BF16 = 1
PISA_SCHEDULE_AUTO = 0
PISA_SCHEDULE_TWO_STAGE = 1
PISA_SCHEDULE_FUSED = 2
PISA_SCHEDULE_SPLIT = 3
PISA_SCORE_LSE = 0
PISA_SCORE_MEAN = 1
PISA_SCORE_MEAN_VAR = 2

PISA_ROPE_HALF = 0
PISA_ROPE_INTERLEAVED = 1
PISA_ROPE_SCALE_NONE = 0
PISA_ROPE_SCALE_LINEAR = 1
PISA_ROPE_SCALE_BASE = 2
PISA_ROPE_SCALE_PARTS = 3
PISA_ROPE_MAX_PAIRS = 64

PISA_OK = 0
PISA_ERR_INVALID_ARG = -1
PISA_ERR_UNSUPPORTED = -2
PISA_ERR_WORKSPACE = -3
PISA_ERR_DEVICE = -4

EXPORTS = (
    "pisa_num_levels", "pisa_pyramid_layout", "pisa_pyramid_bytes",
    "pisa_select_workspace_bytes", "pisa_bsa_workspace_bytes", "pisa_attn_workspace_bytes",
    "pisa_build_pyramid", "pisa_pyramid_append", "pisa_cache_capacity", "pisa_cache_grow", "pisa_select", "pisa_select_static", "pisa_select_flat_bsa",
    "pisa_sparse_attn_fwd", "pisa_attn_union_min_tiles",
    "pisa_attn_bwd_workspace_bytes", "pisa_sparse_attn_bwd",
    "pisa_quality_workspace_bytes", "pisa_selection_quality",
    "pisa_rope_frequencies", "pisa_rope_fwd", "pisa_rope_bwd",
    "pisa_qcache_blocks", "pisa_qcache_bytes", "pisa_qcache_append",
    "pisa_qcache_attn_workspace_bytes", "pisa_qcache_attn_fwd",
    "pisa_profile_enable", "pisa_profile_report", "pisa_status_string", "pisa_last_error",
)


class PisaError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where} failed with status {status}: {detail}")
        self.status = status


class Problem(ctypes.Structure):
    """Mirror of ``pisa_problem``."""
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "H", "Hkv", "Nq", "N", "d", "C", "fanout", "K", "causal", "dtype", "schedule", "Ncap",
                 "score")]

    def __repr__(self):
        return "Problem(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class Strides(ctypes.Structure):
    """Mirror of ``pisa_strides`` (elements)."""
    _fields_ = [("b", ctypes.c_int64), ("h", ctypes.c_int64), ("n", ctypes.c_int64)]


class Rope(ctypes.Structure):
    """Mirror of ``pisa_rope``."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "H", "Hkv", "N", "d", "rot", "layout", "dtype", "pos0", "reserved")]
                + [("pos_bstride", ctypes.c_int64), ("amplitude", ctypes.c_double),
                   ("freq", ctypes.c_double * PISA_ROPE_MAX_PAIRS)])


class QCacheBuffers(ctypes.Structure):
    """Mirror of ``pisa_qcache``."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "k_open", "v_open")]


_DTYPES = {"bf16": PISA_DTYPE_BF16, "f32": PISA_DTYPE_F32,
           torch.bfloat16: PISA_DTYPE_BF16, torch.float32: PISA_DTYPE_F32}
_TORCH = {PISA_DTYPE_BF16: torch.bfloat16, PISA_DTYPE_F32: torch.float32}


def make_problem(B, H, Hkv, Nq, N, d, C, fanout, K, causal=1, dtype="bf16", schedule=PISA_SCHEDULE_AUTO, Ncap=0,
                 score=0):
    """A pisa_problem; Ncap > N reserves rows of k, v and the pyramid for a growing N;
    score picks the selection's block score (PISA_SCORE_LSE / _MEAN / _MEAN_VAR)."""
    return Problem(B, H, Hkv, Nq, N, d, C, fanout, K, int(causal), _DTYPES[dtype], schedule, Ncap, score)


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_31093_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    P = ctypes.POINTER(Problem)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    sig = {
        "pisa_num_levels": (ctypes.c_int, [i32, i32, i32]),
        "pisa_pyramid_layout": (ctypes.c_int, [P, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]),
        "pisa_pyramid_bytes": (sz, [P]),
        "pisa_select_workspace_bytes": (sz, [P]),
        "pisa_bsa_workspace_bytes": (sz, [P]),
        "pisa_attn_workspace_bytes": (sz, [P]),
        "pisa_build_pyramid": (ctypes.c_int, [P, vp, vp, vp]),
        "pisa_pyramid_append": (ctypes.c_int, [P, vp, vp, i32, vp]),
        "pisa_cache_capacity": (ctypes.c_int32, [i32, i32, i32]),
        "pisa_cache_grow": (ctypes.c_int, [P, i32, vp, vp, vp, vp, vp, vp, vp]),
        "pisa_select": (ctypes.c_int, [P, vp, vp, vp, vp, vp, vp, sz, vp]),
        "pisa_select_static": (ctypes.c_int, [P, vp, vp, vp, vp, vp, vp]),
        "pisa_select_flat_bsa": (ctypes.c_int, [P, vp, vp, vp, vp, sz, vp]),
        "pisa_sparse_attn_fwd": (ctypes.c_int, [P, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "pisa_attn_union_min_tiles": (ctypes.c_int, [i32]),
        "pisa_attn_bwd_workspace_bytes": (sz, [P]),
        "pisa_sparse_attn_bwd": (ctypes.c_int, [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "pisa_quality_workspace_bytes": (sz, [P, i32]),
        "pisa_selection_quality": (ctypes.c_int, [P, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]),
        "pisa_rope_frequencies": (ctypes.c_int, [ctypes.POINTER(Rope), ctypes.c_double, i32, ctypes.c_double, i32,
                                                 ctypes.c_double, ctypes.c_double]),
        "pisa_rope_fwd": (ctypes.c_int, [ctypes.POINTER(Rope), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "pisa_rope_bwd": (ctypes.c_int, [ctypes.POINTER(Rope), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "pisa_qcache_blocks": (ctypes.c_int32, [P]),
        "pisa_qcache_bytes": (sz, [P]),
        "pisa_qcache_append": (ctypes.c_int, [P, vp, vp, vp, vp, vp, i32, vp, vp]),
        "pisa_qcache_attn_workspace_bytes": (sz, [P]),
        "pisa_qcache_attn_fwd": (ctypes.c_int, [P, vp, vp, vp, vp, vp, vp, sz, vp]),
        "pisa_profile_enable": (ctypes.c_int, [ctypes.c_int]),
        "pisa_profile_report": (ctypes.c_int, [ctypes.c_char_p, sz]),
        "pisa_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "pisa_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def library():
    """The loaded ctypes.CDLL (its path is ``library()._name``)."""
    return _lib


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _at(x):
    return None if x is None else ctypes.addressof(x)


# the current stream's handle without the Stream object that torch.cuda.current_stream() builds (0.1 us against 2.7)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str):
    if status != PISA_OK:
        raise PisaError(status, where, _lib.pisa_last_error().decode())
    return status


# ------------------------------------------------------------ C entry points ---

def pisa_num_levels(N: int, C: int, fanout: int) -> int:
    L = _lib.pisa_num_levels(N, C, fanout)
    return _check(L, "pisa_num_levels") if L < 0 else L


def pisa_pyramid_layout(p: Problem):
    offs = (ctypes.c_int64 * 64)()
    R = ctypes.c_int64()
    L = _lib.pisa_pyramid_layout(ctypes.byref(p), offs, ctypes.byref(R))
    if L < 0:
        _check(L, "pisa_pyramid_layout")
    return [offs[i] for i in range(L)], R.value


def pisa_pyramid_bytes(p: Problem) -> int:
    return _lib.pisa_pyramid_bytes(ctypes.byref(p))


def pisa_select_workspace_bytes(p: Problem) -> int:
    return _lib.pisa_select_workspace_bytes(ctypes.byref(p))


def pisa_bsa_workspace_bytes(p: Problem) -> int:
    return _lib.pisa_bsa_workspace_bytes(ctypes.byref(p))


def pisa_attn_workspace_bytes(p: Problem) -> int:
    return _lib.pisa_attn_workspace_bytes(ctypes.byref(p))


def pisa_build_pyramid(p: Problem, k, pyramid, stream=None) -> int:
    return _check(_lib.pisa_build_pyramid(ctypes.byref(p), _ptr(k), _ptr(pyramid), _stream(stream)),
                  "pisa_build_pyramid")


def pisa_pyramid_append(p: Problem, k, pyramid, n_old: int, stream=None) -> int:
    return _check(_lib.pisa_pyramid_append(ctypes.byref(p), _ptr(k), _ptr(pyramid), n_old, _stream(stream)),
                  "pisa_pyramid_append")


def pisa_cache_capacity(cap: int, need: int, C: int) -> int:
    r = _lib.pisa_cache_capacity(cap, need, C)
    return _check(r, "pisa_cache_capacity") if r < 0 else r


def pisa_cache_grow(p: Problem, new_cap: int, pyr_old, pyr_new, k_old=None, k_new=None, v_old=None, v_new=None,
                    stream=None) -> int:
    return _check(_lib.pisa_cache_grow(ctypes.byref(p), new_cap, _ptr(pyr_old), _ptr(pyr_new), _ptr(k_old), _ptr(k_new),
                                       _ptr(v_old), _ptr(v_new), _stream(stream)), "pisa_cache_grow")


def pisa_select(p: Problem, q, k, pyramid, block_idx, block_score=None, ws=None, ws_bytes=0, stream=None) -> int:
    return _check(_lib.pisa_select(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(pyramid), _ptr(block_idx),
                                   _ptr(block_score), _ptr(ws), ws_bytes, _stream(stream)), "pisa_select")


def pisa_select_static(p: Problem, q, k, pyramid, block_idx, block_score=None, stream=None) -> int:
    return _check(_lib.pisa_select_static(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(pyramid), _ptr(block_idx),
                                          _ptr(block_score), _stream(stream)), "pisa_select_static")


PISA_STATIC_SCRATCH_BYTES = 32 << 20  # include/pisa.h


def pisa_select_flat_bsa(p: Problem, q, pyramid, block_idx, ws=None, ws_bytes=0, stream=None) -> int:
    return _check(_lib.pisa_select_flat_bsa(ctypes.byref(p), _ptr(q), _ptr(pyramid), _ptr(block_idx),
                                            _ptr(ws), ws_bytes, _stream(stream)), "pisa_select_flat_bsa")


def pisa_sparse_attn_fwd(p: Problem, q, k, v, block_idx, o, lse=None, ws=None, ws_bytes=0, stream=None) -> int:
    return _check(_lib.pisa_sparse_attn_fwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx),
                                            _ptr(o), _ptr(lse), _ptr(ws), ws_bytes, _stream(stream)),
                  "pisa_sparse_attn_fwd")


def pisa_attn_bwd_workspace_bytes(p: Problem) -> int:
    return _lib.pisa_attn_bwd_workspace_bytes(ctypes.byref(p))


def pisa_sparse_attn_bwd(p: Problem, q, k, v, block_idx, o, lse, d_o, dq, dk, dv, ws=None, ws_bytes=0,
                         stream=None) -> int:
    return _check(_lib.pisa_sparse_attn_bwd(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx), _ptr(o),
                                            _ptr(lse), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), ws_bytes,
                                            _stream(stream)), "pisa_sparse_attn_bwd")


def pisa_quality_workspace_bytes(p: Problem, n_rows: int) -> int:
    return _lib.pisa_quality_workspace_bytes(ctypes.byref(p), n_rows)


def pisa_selection_quality(p: Problem, q, k, block_idx, rows, n_rows: int, metrics, ref_idx=None, ws=None,
                           ws_bytes=0, stream=None) -> int:
    return _check(_lib.pisa_selection_quality(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(block_idx), _ptr(rows), n_rows,
                                              _ptr(metrics), _ptr(ref_idx), _ptr(ws), ws_bytes, _stream(stream)),
                  "pisa_selection_quality")


def pisa_rope_frequencies(r: Rope, base: float, scaling: int, factor: float, ctx: int, fast: float, slow: float) -> int:
    return _check(_lib.pisa_rope_frequencies(ctypes.byref(r), base, scaling, factor, ctx, fast, slow),
                  "pisa_rope_frequencies")


def _rope_call(fn, name, r, q, qs, k, ks, positions, qo, qos, ko, kos, stream):
    return _check(fn(ctypes.byref(r), _ptr(q), _at(qs), _ptr(k), _at(ks), _ptr(positions), _ptr(qo), _at(qos), _ptr(ko),
                     _at(kos), _stream(stream)), name)


def pisa_rope_fwd(r: Rope, q, q_strides, k, k_strides, positions, q_out, q_out_strides, k_out, k_out_strides,
                  stream=None) -> int:
    return _rope_call(_lib.pisa_rope_fwd, "pisa_rope_fwd", r, q, q_strides, k, k_strides, positions, q_out, q_out_strides, k_out,
                      k_out_strides, stream)


def pisa_rope_bwd(r: Rope, d_q_out, d_q_out_strides, d_k_out, d_k_out_strides, positions, d_q, d_q_strides, d_k,
                  d_k_strides, stream=None) -> int:
    return _rope_call(_lib.pisa_rope_bwd, "pisa_rope_bwd", r, d_q_out, d_q_out_strides, d_k_out, d_k_out_strides, positions, d_q, d_q_strides,
                      d_k, d_k_strides, stream)


def pisa_qcache_blocks(p: Problem) -> int:
    M = _lib.pisa_qcache_blocks(ctypes.byref(p))
    return _check(M, "pisa_qcache_blocks") if M < 0 else M


def pisa_qcache_bytes(p: Problem) -> int:
    return _lib.pisa_qcache_bytes(ctypes.byref(p))


def pisa_qcache_append(p: Problem, cache, k_new, k_strides, v_new, v_strides, n_old: int, pyramid=None,
                       stream=None) -> int:
    return _check(_lib.pisa_qcache_append(ctypes.byref(p), cache.address, _ptr(k_new), _at(k_strides), _ptr(v_new),
                                          _at(v_strides), n_old, _ptr(pyramid), _stream(stream)), "pisa_qcache_append")


def pisa_qcache_attn_workspace_bytes(p: Problem) -> int:
    return _lib.pisa_qcache_attn_workspace_bytes(ctypes.byref(p))


def pisa_qcache_attn_fwd(p: Problem, cache, q, block_idx, o, lse=None, ws=None, ws_bytes=0, stream=None) -> int:
    return _check(_lib.pisa_qcache_attn_fwd(ctypes.byref(p), cache.address, _ptr(q), _ptr(block_idx), _ptr(o), _ptr(lse),
                                            _ptr(ws), ws_bytes, _stream(stream)), "pisa_qcache_attn_fwd")


def pisa_attn_union_min_tiles(n: int) -> int:
    """Sets the row-tile union threshold of pisa_sparse_attn_fwd (n < 0: off); returns the previous one."""
    return _lib.pisa_attn_union_min_tiles(int(n))


def pisa_profile_enable(on: bool) -> int:
    return _lib.pisa_profile_enable(1 if on else 0)


def pisa_profile_report() -> dict:
    """{kernel: (launches, total_ms)} since the last report (waits for the events)."""
    cap = 1 << 16
    buf = ctypes.create_string_buffer(cap)
    _lib.pisa_profile_report(buf, cap)
    out = {}
    for line in buf.value.decode().splitlines():
        name, cnt, ms = line.split()
        out[name] = (int(cnt), float(ms))
    return out


def pisa_status_string(status: int) -> str:
    return _lib.pisa_status_string(status).decode()


def pisa_last_error() -> str:
    return _lib.pisa_last_error().decode()


# ----------------------------------------------- allocation-side conveniences ---

def _workspace(nbytes: int, device):
    if nbytes == 0:
        return None
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


_HERE = contextlib.nullcontext()


def _elsewhere(stream):
    return stream is not None and _stream(stream) != _stream(None)


def _on(stream, device):
    """Context in which what a call on `stream` uses is allocated: memory of the current stream's would be handed to its
    next allocations while `stream` still works on it, and may be in use there when `stream` begins."""
    if not _elsewhere(stream):
        return _HERE
    return torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device=device))


def _results(stream, *tensors):
    """Outputs allocated under _on, which the caller's stream reads: not handed on before it has."""
    if _elsewhere(stream):
        for x in tensors:
            if x is not None:
                x.record_stream(torch.cuda.current_stream(x.device))
    return tensors if len(tensors) > 1 else tensors[0]


def build_pyramid(p: Problem, k, stream=None):
    """Allocate [B, Hkv, R, d] float32 and fill it with pisa_build_pyramid."""
    _, R = pisa_pyramid_layout(p)
    with _on(stream, k.device):
        pyr = torch.empty((p.B, p.Hkv, R, p.d), dtype=torch.float32, device=k.device)
    pisa_build_pyramid(p, k, pyr, stream)
    return _results(stream, pyr)


def grow_cache(p: Problem, new_cap: int, pyramid, k=None, v=None, stream=None):
    """Allocate buffers for new_cap tokens and move the cache of problem p into
    them with pisa_cache_grow.  Returns (problem with Ncap = new_cap, pyramid,
    k, v); k and v are None when not given."""
    pn = Problem(*[getattr(p, n) for n, _ in Problem._fields_])
    pn.Ncap = new_cap
    _, R = pisa_pyramid_layout(pn)
    kn = vn = None
    with _on(stream, pyramid.device):
        pyr = torch.empty((p.B, p.Hkv, R, p.d), dtype=torch.float32, device=pyramid.device)
        if k is not None:
            kn = torch.empty((p.B, p.Hkv, new_cap, p.d), dtype=k.dtype, device=k.device)
            vn = torch.empty((p.B, p.Hkv, new_cap, p.d), dtype=v.dtype, device=v.device)
    pisa_cache_grow(p, new_cap, pyramid, pyr, k, kn, v, vn, stream)
    return pn, *_results(stream, pyr, kn, vn)


def select(p: Problem, q, k, pyramid, with_score=False, stream=None):
    """Allocate outputs and workspace, run pisa_select; returns idx (and scores)."""
    nb = pisa_select_workspace_bytes(p)
    with _on(stream, q.device):
        idx = torch.empty((p.B, p.Hkv, p.Nq, p.K), dtype=torch.int32, device=q.device)
        sc = torch.empty((p.B, p.Hkv, p.Nq, p.K), dtype=torch.float32, device=q.device) if with_score else None
        ws = _workspace(nb, q.device)
    pisa_select(p, q, k, pyramid, idx, sc, ws, nb, stream)
    _results(stream, idx, sc)
    return (idx, sc) if with_score else idx


def select_flat_bsa(p: Problem, q, pyramid, stream=None):
    nb = pisa_bsa_workspace_bytes(p)
    with _on(stream, q.device):
        idx = torch.empty((p.B, p.Hkv, p.Nq, p.K), dtype=torch.int32, device=q.device)
        ws = _workspace(nb, q.device)
    pisa_select_flat_bsa(p, q, pyramid, idx, ws, nb, stream)
    return _results(stream, idx)


def sparse_attn_fwd(p: Problem, q, k, v, block_idx, stream=None):
    nb = pisa_attn_workspace_bytes(p)
    with _on(stream, q.device):
        o = torch.empty_like(q)
        lse = torch.empty((p.B, p.H, p.Nq), dtype=torch.float32, device=q.device)
        ws = _workspace(nb, q.device)
    pisa_sparse_attn_fwd(p, q, k, v, block_idx, o, lse, ws, nb, stream)
    return _results(stream, o, lse)


def selection_quality(p: Problem, q, k, block_idx, rows, stream=None):
    """Allocate outputs and workspace, run pisa_selection_quality on the listed
    rows (a device int32 tensor); returns (metrics [B,Hkv,n,3], ref [B,Hkv,n,K])."""
    n = int(rows.numel())
    nb = pisa_quality_workspace_bytes(p, n)
    with _on(stream, q.device):
        met = torch.empty((p.B, p.Hkv, n, 3), dtype=torch.float32, device=q.device)
        ref = torch.empty((p.B, p.Hkv, n, p.K), dtype=torch.int32, device=q.device)
        ws = _workspace(nb, q.device)
    pisa_selection_quality(p, q, k, block_idx, rows, n, met, ref, ws, nb, stream)
    return _results(stream, met, ref)


def sparse_attn_bwd(p: Problem, q, k, v, block_idx, o, lse, d_o, stream=None):
    """Allocate gradients and workspace, run pisa_sparse_attn_bwd; returns (dq, dk, dv)."""
    nb = pisa_attn_bwd_workspace_bytes(p)
    with _on(stream, q.device):
        dq = torch.empty_like(q)
        dk = torch.empty_like(k)
        dv = torch.empty_like(v)
        ws = _workspace(nb, q.device)
    pisa_sparse_attn_bwd(p, q, k, v, block_idx, o, lse, d_o, dq, dk, dv, ws, nb, stream)
    return _results(stream, dq, dk, dv)


# ------------------------------------------------- rotary positions, 8-bit cache ---

_LAYOUTS = {"half": PISA_ROPE_HALF, "interleaved": PISA_ROPE_INTERLEAVED}
_SCALINGS = {"none": PISA_ROPE_SCALE_NONE, "linear": PISA_ROPE_SCALE_LINEAR, "base": PISA_ROPE_SCALE_BASE,
             "parts": PISA_ROPE_SCALE_PARTS}


def _refuse(x, name, dtype, shape, device, contiguous=True):
    raise ValueError(f"{name}: expected {'a contiguous ' if contiguous else ''}{dtype} {tuple(shape)} on the current device "
                     f"(cuda:{device}), got {x.dtype} {tuple(x.shape)} (strides {x.stride()}) on {x.device}")


def _take(x, name, dtype, shape, device):
    """x, a contiguous tensor of device number `device` with this dtype and shape; ValueError otherwise."""
    if x.dtype != dtype or x.shape != shape or x.get_device() != device or not x.is_contiguous():
        _refuse(x, name, dtype, shape, device)
    return x


@functools.lru_cache(maxsize=256)
def _strides(b, h, n):
    return Strides(b, h, n)


def _strided(x, name, dtype, shape, device):
    """The pisa_strides of a [B, heads, rows, d] tensor (None where it is contiguous)."""
    if x.dtype != dtype or x.shape != shape or x.get_device() != device:
        _refuse(x, name, dtype, shape, device, contiguous=False)
    if x.is_contiguous():
        return None
    b, h, n, one = x.stride()
    if one != 1:
        raise ValueError(f"{name}: its last dimension must be contiguous (strides {x.stride()})")
    # the stride of a dimension of one entry is never used
    return _strides(b if shape[0] > 1 else 0, h if shape[1] > 1 else 0, n if shape[2] > 1 else 0)


def make_rope(B, H, Hkv, N, d, rot=None, layout="half", dtype="bf16", base=10000.0, scaling="none", factor=1.0, ctx=4096,
              fast=32.0, slow=1.0, pos0=0):
    """A pisa_rope with the frequencies of pisa_rope_frequencies; rot defaults to d."""
    r = Rope(B, H, Hkv, N, d, d if rot is None else rot, _LAYOUTS[layout], _DTYPES[dtype], pos0, 0, 0, 1.0)
    pisa_rope_frequencies(r, base, _SCALINGS[scaling], factor, ctx, fast, slow)
    return r


def _side(x, y, name, dtype, shape, device, stream):
    """(x, its strides, output, its strides) of one side of a rotation, the output allocated where y is None."""
    if x is None:
        if y is not None:
            raise ValueError(f"{name}_out without {name}")
        return None, None, None, None
    xs = _strided(x, name, dtype, shape, device)
    if y is None:
        with _on(stream, x.device):
            y = torch.empty(shape, dtype=dtype, device=x.device)
        return x, xs, _results(stream, y), None
    return x, xs, y, _strided(y, name + "_out", dtype, shape, device)


def _rope(turn, r: Rope, q, k, positions, q_out, k_out, stream):
    dt, dev, B, N, d = _TORCH[r.dtype], torch.cuda.current_device(), r.B, r.N, r.d
    if positions is not None:
        shared = positions.dim() == 1
        _take(positions, "positions", torch.int32, (N,) if shared else (B, N), dev)
        stride = 0 if shared else N
        if r.pos_bstride != stride:  # in a copy: the caller's may be in use by another thread's call
            r = Rope.from_buffer_copy(r)
            r.pos_bstride = stride
    q, qs, q_out, qos = _side(q, q_out, "q", dt, (B, r.H, N, d), dev, stream)
    k, ks, k_out, kos = _side(k, k_out, "k", dt, (B, r.Hkv, N, d), dev, stream)
    turn(r, q, qs, k, ks, positions, q_out, qos, k_out, kos, stream)
    return q_out, k_out


def rope_fwd(r: Rope, q, k=None, positions=None, q_out=None, k_out=None, stream=None):
    """Turn q [B, H, N, d] and k [B, Hkv, N, d] (views with a contiguous last dimension; either may be None)
    by their positions (int32 [N] or [B, N]; default pos0, pos0 + 1, ...).  Returns (q_out, k_out), allocated
    contiguous where not given."""
    return _rope(pisa_rope_fwd, r, q, k, positions, q_out, k_out, stream)


def rope_bwd(r: Rope, d_q_out, d_k_out=None, positions=None, d_q=None, d_k=None, stream=None):
    """The gradients of rope_fwd's inputs from those of its outputs; tensors as there."""
    return _rope(pisa_rope_bwd, r, d_q_out, d_k_out, positions, d_q, d_k, stream)


class QCache:
    """The buffers of an 8-bit key/value cache (pisa_qcache): uint8 codes k [B, Hkv, M, C, d] and v [B, Hkv, M, d, C],
    float32 scales [B, Hkv, M], and for appending the raw rows of the last block, [B, Hkv, C, d]."""

    def __init__(self, k, v, k_scale, v_scale, k_open=None, v_open=None):
        B, H, M, C, d = k.shape
        dev = k.get_device()
        if dev < 0:
            raise ValueError(f"the cache lives on a GPU, got {k.device}")
        _take(k, "k", torch.uint8, (B, H, M, C, d), dev)
        _take(v, "v", torch.uint8, (B, H, M, d, C), dev)
        _take(k_scale, "k_scale", torch.float32, (B, H, M), dev)
        _take(v_scale, "v_scale", torch.float32, (B, H, M), dev)
        if (k_open is None) != (v_open is None):
            raise ValueError("k_open and v_open come together")
        if k_open is not None:
            _take(k_open, "k_open", k_open.dtype, (B, H, C, d), dev)
            _take(v_open, "v_open", k_open.dtype, (B, H, C, d), dev)
        self.k, self.v, self.k_scale, self.v_scale, self.k_open, self.v_open = k, v, k_scale, v_scale, k_open, v_open
        self.device, self._shape = dev, (B, H, M, C, d)
        self._c = QCacheBuffers(*(_ptr(x) for x in (k, v, k_scale, v_scale, k_open, v_open)))
        self.address = ctypes.addressof(self._c)

    def check(self, p: Problem, appending=False):
        """ValueError unless this is a cache of problem p on the current device."""
        B, H, M, C, d = self._shape
        if (B, H, C, d) != (p.B, p.Hkv, p.C, p.d) or M != -(-(p.Ncap or p.N) // C):
            raise ValueError(f"the cache's codes {self._shape} do not fit {p}")
        if self.device != torch.cuda.current_device():
            raise ValueError(f"the cache is on cuda:{self.device}, the current device is cuda:{torch.cuda.current_device()}")
        if appending and (self.k_open is None or self.k_open.dtype != _TORCH[p.dtype]):
            raise ValueError("appending needs k_open and v_open in the problem's dtype")


def make_qcache(p: Problem, device=None):
    """An empty cache for problem p (reserving Ncap tokens), cleared on the current stream."""
    M, dev = pisa_qcache_blocks(p), torch.device("cuda", torch.cuda.current_device()) if device is None else device
    new = dict(device=dev)
    k = torch.zeros((p.B, p.Hkv, M, p.C, p.d), dtype=torch.uint8, **new)
    v = torch.zeros((p.B, p.Hkv, M, p.d, p.C), dtype=torch.uint8, **new)
    scales = (torch.ones((p.B, p.Hkv, M), dtype=torch.float32, **new) for _ in range(2))
    raw = (torch.zeros((p.B, p.Hkv, p.C, p.d), dtype=_TORCH[p.dtype], **new) for _ in range(2))
    return QCache(k, v, *scales, *raw)


def grow_qcache(p: Problem, new_cap: int, cache: QCache, pyramid=None):
    """Allocate a cache for new_cap tokens and move problem p's into it (on the current stream), its pyramid with
    pisa_cache_grow.  Returns (problem with Ncap = new_cap, cache, pyramid); pyramid is None when not given."""
    cache.check(p)
    pn = Problem(*[getattr(p, n) for n, _ in Problem._fields_])
    pn.Ncap = new_cap
    if new_cap < (p.Ncap or p.N):
        raise ValueError(f"new_cap ({new_cap}) is below the current capacity ({p.Ncap or p.N})")
    new, M = make_qcache(pn), -(-p.N // p.C)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(new, name)[:, :, :M].copy_(getattr(cache, name)[:, :, :M])
    if cache.k_open is not None:
        new.k_open.copy_(cache.k_open)
        new.v_open.copy_(cache.v_open)
    return pn, new, None if pyramid is None else grow_cache(p, new_cap, pyramid)[1]


def qcache_append(p: Problem, cache: QCache, k_new, v_new, n_old: int, pyramid=None, stream=None):
    """Append rows n_old .. N-1 (k_new, v_new: [B, Hkv, N - n_old, d], views with a contiguous last dimension) to
    the cache, and bring the pyramid with it where one is given.  A smaller n_old than before takes rows back: in the last
    block or on a block's border as it is; after a draft that passed a border only with cache.k_open and cache.v_open put
    back as they were before it."""
    cache.check(p, appending=True)
    shape, dt, dev = (p.B, p.Hkv, p.N - n_old, p.d), _TORCH[p.dtype], cache.device
    ks, vs = _strided(k_new, "k_new", dt, shape, dev), _strided(v_new, "v_new", dt, shape, dev)
    if pyramid is not None:
        _take(pyramid, "pyramid", torch.float32, (p.B, p.Hkv, pyramid.shape[2], p.d), dev)
        if pyramid.numel() * 4 != pisa_pyramid_bytes(p):
            raise ValueError(f"pyramid: {tuple(pyramid.shape)} does not fit {p}")
    pisa_qcache_append(p, cache, k_new, ks, v_new, vs, n_old, pyramid, stream)


def qcache_attn_fwd(p: Problem, cache: QCache, q, block_idx, stream=None):
    """Allocate outputs and workspace, run pisa_qcache_attn_fwd; returns (o, lse)."""
    cache.check(p)
    dev = cache.device
    _take(q, "q", _TORCH[p.dtype], (p.B, p.H, p.Nq, p.d), dev)
    _take(block_idx, "block_idx", torch.int32, (p.B, p.Hkv, p.Nq, p.K), dev)
    nb = pisa_qcache_attn_workspace_bytes(p)
    with _on(stream, q.device):
        o = torch.empty_like(q)
        lse = torch.empty((p.B, p.H, p.Nq), dtype=torch.float32, device=q.device)
        ws = _workspace(nb, q.device)
    pisa_qcache_attn_fwd(p, cache, q, block_idx, o, lse, ws, nb, stream)
    return _results(stream, o, lse)
