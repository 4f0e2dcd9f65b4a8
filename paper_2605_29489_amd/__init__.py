"""Python binding of libmergepipe.so (budgeted weight-space merging on MI355X).

Argument marshalling only: every step of the path (index, plan, merge) runs
in the library's HIP kernels.  PyTorch is used for device/pinned memory and
streams.  The functions have the names of the C entry points declared in
``include/mergepipe.h``; they take torch tensors and raise ``MPError`` on a
non-zero status.

The library must have been built (``python -m paper_2605_29489_amd.build``
or ``__graft_entry__.build()``); importing this package without it raises
ImportError -- there is no fallback.
"""

from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmergepipe.so")

MP_OK = 0
MP_E_ARG = -1
MP_E_UNSUPPORTED = -2
MP_E_NOMEM = -3
MP_E_HIP = -4
MP_E_IO = -5
MP_F32, MP_BF16 = 0, 1
MP_DEVICE, MP_HOST_PINNED, MP_HOST_PAGEABLE, MP_HOST_FILE = 0, 1, 2, 3
MP_EXPERTS_DELTA = 16  # OR-ed into residency: experts hold W_i - W_0
MP_COMBINE_LINEAR, MP_COMBINE_SIGN_ELECT = 0, 1
MP_PLAN_PER_BYTE, MP_PLAN_SKIP_ZERO = 1, 2
MP_ACT_NONE, MP_ACT_RELU, MP_ACT_GELU, MP_ACT_GELU_TANH, MP_ACT_SILU = range(5)
MP_NORM_RMS = 1
MP_MOE_RENORM = 1
MP_ROPE_INTERLEAVED = 1
MP_ROPE_PLAIN, MP_ROPE_LINEAR, MP_ROPE_NTK, MP_ROPE_PARTS, MP_ROPE_YARN = range(5)

EXPORTS = ("mp_layout_blocks", "mp_index_blocks", "mp_index_ties", "mp_ties_tensor_thresholds", "mp_plan",
           "mp_plan_noalloc", "mp_coverage", "mp_merge_avg", "mp_merge_avg_renorm",
           "mp_merge_ties",
           "mp_merge_ties_tau", "mp_merge_dare", "mp_lora_materialize", "mp_lora_merge_ties_tau", "mp_stream_copy",
           "mp_linear", "mp_linear_backward", "mp_linear_workspace", "mp_norm", "mp_norm_backward",
           "mp_norm_workspace", "mp_moe", "mp_moe_workspace",
           "mp_rope", "mp_rope_backward", "mp_rope_frequencies", "mp_kv_append", "mp_kv_attend",
           "mp_kv_attend_workspace",
           "mp_set_stage_bytes",
           "mp_set_workspace_limit", "mp_workspace_bytes", "mp_ties_tensor_left", "mp_last_error", "mp_release")


class mp_layout(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("dtype", C.c_int32),
                ("numel", C.POINTER(C.c_int64)), ("block_elems", C.c_int64)]


class mp_plan_stats(C.Structure):
    _fields_ = [("budget_bytes", C.c_uint64), ("cost_bytes", C.c_uint64), ("full_bytes", C.c_uint64),
                ("n_selected", C.c_uint64), ("n_units", C.c_uint64), ("digest", C.c_uint64)]

    def as_dict(self):
        return {f: int(getattr(self, f)) for f, _ in self._fields_}


class mp_io_stats(C.Structure):
    _fields_ = [("expert_bytes", C.c_uint64), ("base_bytes", C.c_uint64), ("out_bytes", C.c_uint64),
                ("h2d_bytes", C.c_uint64), ("expert_bytes_by_expert", C.c_uint64 * 32)]

    def as_dict(self):
        d = {f: int(getattr(self, f)) for f, _ in self._fields_[:4]}
        d["expert_bytes_by_expert"] = [int(x) for x in self.expert_bytes_by_expert]
        return d


class mp_lora_tensor(C.Structure):
    _fields_ = [("tensor", C.c_int32), ("rank", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("a_off", C.c_int64), ("b_off", C.c_int64), ("scale", C.c_float)]


class mp_linear_shape(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32)] + [
        (n, C.c_int64) for n in ("m", "n", "k", "ldx", "ldw", "ldy", "ldz", "ldr")]


class mp_norm_shape(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("flags", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("ldx", C.c_int64), ("ldy", C.c_int64), ("eps", C.c_float)]


class mp_moe_layer(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("top_k", C.c_int32), ("flags", C.c_int32)] + [
        (n, C.c_int64) for n in ("hidden", "ffn", "gate_off", "up_off", "down_off")]


class mp_rope_shape(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("flags", C.c_int32)] + [
        (n, C.c_int64) for n in ("tokens", "heads", "head_dim", "rot_dim", "ldx", "hdx", "ldy", "hdy")] + [
        ("amplitude", C.c_float)]


class mp_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32)] + [(n, C.c_double) for n in ("base", "factor", "original", "low", "high")]


class mp_kv_cache(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("flags", C.c_int32)] + [
        (n, C.c_int64) for n in ("pages", "page_size", "heads", "head_dim", "page_stride", "slot_stride",
                                 "head_stride")] + [("k", C.c_void_p), ("v", C.c_void_p)]


class mp_kv_rows(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("q_heads", C.c_int64), ("rot_dim", C.c_int64), ("flags", C.c_int32),
                ("amplitude", C.c_float)] + [(n, C.c_int64) for n in ("ldk", "ldv", "ldq", "ldqo")]


class mp_kv_attend_shape(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("rows", "q_heads", "width", "ldq", "ldo", "ldt", "window")] + [
        ("scale", C.c_float)]


class MPError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"mergepipe error {code}: {msg}")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
    # Buffers come from torch, which ships its own HIP runtime.  Load that one
    # first, so this library binds to the same runtime: loaded the other way
    # round, the library's runtime does not know torch's allocations.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = C.CDLL(LIB_PATH)
    vp, i32, u32, u64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64
    lp = C.POINTER(mp_layout)
    L.mp_layout_blocks.argtypes = [lp, C.POINTER(C.c_int64)]
    L.mp_index_blocks.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, vp]
    L.mp_index_ties.argtypes = [lp, vp, C.POINTER(vp), i32, i32, C.c_double, vp, vp, vp]
    L.mp_plan.argtypes = [lp, i32, vp, C.POINTER(C.c_float), u64, u32, vp, C.POINTER(mp_plan_stats), vp]
    L.mp_plan_noalloc.argtypes = L.mp_plan.argtypes
    L.mp_merge_avg.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, C.POINTER(C.c_float), vp,
                               C.POINTER(mp_io_stats), vp]
    L.mp_merge_avg_renorm.argtypes = L.mp_merge_avg.argtypes
    L.mp_coverage.argtypes = [lp, i32, vp, C.POINTER(C.c_uint64), vp]
    L.mp_ties_tensor_thresholds.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, C.c_double, vp, vp]
    L.mp_merge_ties.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, C.c_double, C.c_float, vp,
                                C.POINTER(mp_io_stats), vp]
    L.mp_merge_ties_tau.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, vp, C.c_float, vp,
                                    C.POINTER(mp_io_stats), vp]
    L.mp_merge_dare.argtypes = [lp, vp, C.POINTER(vp), i32, i32, vp, C.c_double, u32, i32,
                                C.POINTER(C.c_float), C.c_float, vp, C.POINTER(mp_io_stats), vp]
    L.mp_lora_materialize.argtypes = [lp, C.POINTER(mp_lora_tensor), i32, C.POINTER(vp), i32, vp, C.POINTER(vp),
                                      vp]
    L.mp_lora_merge_ties_tau.argtypes = [lp, vp, C.POINTER(mp_lora_tensor), i32, C.POINTER(vp), i32, vp, vp,
                                         C.c_float, vp, vp]
    i64, lsp, nsp, mlp = C.c_int64, C.POINTER(mp_linear_shape), C.POINTER(mp_norm_shape), C.POINTER(mp_moe_layer)
    L.mp_linear.argtypes = [lsp, vp, vp, vp, vp, vp, vp, vp, u64, vp]
    L.mp_linear_backward.argtypes = [lsp, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, u64, vp]
    L.mp_linear_workspace.argtypes = [lsp, i32, C.POINTER(u64)]
    L.mp_norm.argtypes = [nsp, vp, vp, vp, vp, vp, vp, vp]
    L.mp_norm_backward.argtypes = [nsp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, u64, vp]
    L.mp_norm_workspace.argtypes = [nsp, C.POINTER(u64)]
    L.mp_moe.argtypes = [mlp, i64, vp, i64, vp, vp, C.POINTER(vp), i32, i32, vp, i64, vp, i64, vp, vp, vp, u64, vp]
    L.mp_moe_workspace.argtypes = [mlp, i64, C.POINTER(u64)]
    rsp, kcp, asp = C.POINTER(mp_rope_shape), C.POINTER(mp_kv_cache), C.POINTER(mp_kv_attend_shape)
    L.mp_rope.argtypes = L.mp_rope_backward.argtypes = [rsp, vp, vp, vp, vp, vp]
    L.mp_rope_frequencies.argtypes = [C.POINTER(mp_rope_scaling), i64, C.POINTER(C.c_double), C.POINTER(C.c_float)]
    L.mp_kv_append.argtypes = [kcp, C.POINTER(mp_kv_rows), vp, vp, vp, vp, vp, vp, vp, vp]
    L.mp_kv_attend.argtypes = [kcp, asp, vp, vp, vp, vp, vp, vp, u64, vp]
    L.mp_kv_attend_workspace.argtypes = [kcp, asp, C.POINTER(u64)]
    L.mp_last_error.restype = C.c_char_p
    L.mp_stream_copy.argtypes = [vp, vp, u64, vp]
    L.mp_set_stage_bytes.argtypes = [u64]
    L.mp_set_stage_bytes.restype = i32
    L.mp_set_workspace_limit.argtypes = [u64]
    L.mp_set_workspace_limit.restype = i32
    L.mp_workspace_bytes.argtypes = []
    L.mp_workspace_bytes.restype = u64
    L.mp_ties_tensor_left.argtypes = []
    L.mp_ties_tensor_left.restype = C.c_int64
    L.mp_last_error.argtypes = []
    L.mp_release.argtypes = []
    for name in ("mp_layout_blocks", "mp_index_blocks", "mp_index_ties", "mp_ties_tensor_thresholds", "mp_plan",
                 "mp_plan_noalloc", "mp_coverage", "mp_merge_avg",
                 "mp_merge_avg_renorm", "mp_merge_ties",
                 "mp_merge_ties_tau",
                 "mp_merge_dare", "mp_lora_materialize", "mp_lora_merge_ties_tau", "mp_stream_copy",
                 "mp_linear", "mp_linear_backward", "mp_linear_workspace", "mp_norm", "mp_norm_backward",
                 "mp_norm_workspace", "mp_moe", "mp_moe_workspace",
                 "mp_rope", "mp_rope_backward", "mp_rope_frequencies", "mp_kv_append", "mp_kv_attend",
                 "mp_kv_attend_workspace"):
        getattr(L, name).restype = C.c_int
    return L


lib = _load()


@dataclass
class Layout:
    """Host-side mp_layout: tensor numels, block size and dtype code."""

    numel: Sequence[int]
    block_elems: int
    dtype: int  # MP_F32 or MP_BF16

    def __post_init__(self):
        self._numel = (C.c_int64 * max(len(self.numel), 1))(*[int(n) for n in self.numel])
        self._s = mp_layout(len(self.numel), int(self.dtype), C.cast(self._numel, C.POINTER(C.c_int64)),
                            int(self.block_elems))

    @property
    def ref(self):
        return C.byref(self._s)

    @property
    def elem_bytes(self) -> int:
        return 4 if self.dtype == MP_F32 else 2

    @property
    def n_params(self) -> int:
        return int(sum(int(n) for n in self.numel))


def _check(rc: int):
    if rc != MP_OK:
        raise MPError(rc, lib.mp_last_error().decode())


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _ptrs(ts):
    """Array of expert pointers: tensors by address, file paths (MP_HOST_FILE)
    as NUL-terminated strings kept alive with the array."""
    keep, vals = [], []
    for t in ts:
        if isinstance(t, (str, bytes, os.PathLike)):
            b = C.create_string_buffer(os.fsencode(t))
            keep.append(b)
            vals.append(C.addressof(b))
        else:
            vals.append(_ptr(t))
    arr = (C.c_void_p * max(len(ts), 1))(*vals)
    arr._keep = keep
    return arr


def _floats(xs, K):
    if xs is None:
        return None
    xs = [float(x) for x in xs]
    if len(xs) != K:
        raise ValueError(f"expected {K} coefficients, got {len(xs)}")
    return (C.c_float * K)(*xs)


@functools.lru_cache(maxsize=None)
def _raw_stream():
    """torch's call for the current stream's handle alone (0.3 us against 3), and that for the current device."""
    import torch
    return getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device


def _stream(stream):
    if stream is None:
        raw, device = _raw_stream()
        if raw is not None:
            return raw(device())
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return C.c_void_p(stream)
    return C.c_void_p(stream.cuda_stream)


def mp_layout_blocks(layout: Layout) -> int:
    g = C.c_int64(0)
    _check(lib.mp_layout_blocks(layout.ref, C.byref(g)))
    return int(g.value)


def mp_index_blocks(layout: Layout, base, experts, sumsq, residency: int = MP_DEVICE, stream=None,
                    delta: bool = False):
    _check(lib.mp_index_blocks(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta),
                               _ptr(sumsq), _stream(stream)))


def mp_index_ties(layout: Layout, base, experts, density: float, tau, sumsq=None, residency: int = MP_DEVICE,
                  stream=None, delta: bool = False):
    """Per-unit TIES thresholds (uint32 patterns in `tau`, G*K) and, if given, sumsq."""
    _check(lib.mp_index_ties(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta),
                             float(density),
                             _ptr(sumsq), _ptr(tau), _stream(stream)))


def mp_plan(layout: Layout, K: int, sumsq, w, budget_bytes: int, mask, flags: int = 0, stream=None) -> dict:
    st = mp_plan_stats()
    _check(lib.mp_plan(layout.ref, K, _ptr(sumsq), _floats(w, K), int(budget_bytes), flags, _ptr(mask),
                       C.byref(st), _stream(stream)))
    return st.as_dict()


def mp_plan_noalloc(layout: Layout, K: int, sumsq, w, budget_bytes: int, mask, flags: int = 0,
                    stream=None) -> dict:
    """mp_plan on the library's fixed device array (allocates nothing)."""
    st = mp_plan_stats()
    _check(lib.mp_plan_noalloc(layout.ref, K, _ptr(sumsq), _floats(w, K), int(budget_bytes), flags, _ptr(mask),
                               C.byref(st), _stream(stream)))
    return st.as_dict()


def _res(residency: int, delta: bool) -> int:
    return residency | (MP_EXPERTS_DELTA if delta else 0)


def _io(io):
    return C.byref(io) if io is not None else None


def mp_ties_tensor_thresholds(layout: Layout, base, experts, mask, density: float, tau,
                              residency: int = MP_DEVICE, stream=None, delta: bool = False):
    """Per-unit TIES thresholds at tensor scope for this mask (device uint32 [G*K])."""
    _check(lib.mp_ties_tensor_thresholds(layout.ref, _ptr(base), _ptrs(experts), len(experts),
                                         _res(residency, delta), _ptr(mask), float(density), _ptr(tau),
                                         _stream(stream)))


def mp_coverage(layout: Layout, K: int, mask, stream=None):
    """Touched elements per (tensor, expert) of a mask: numpy uint64 [n_tensors, K]."""
    import numpy as np
    cov = np.zeros(len(layout.numel) * K, np.uint64)
    _check(lib.mp_coverage(layout.ref, K, _ptr(mask), cov.ctypes.data_as(C.POINTER(C.c_uint64)), _stream(stream)))
    return cov.reshape(len(layout.numel), K)


def mp_merge_avg(layout: Layout, base, experts, mask, alpha, out, residency: int = MP_DEVICE,
                 io: bool = False, stream=None, delta: bool = False) -> Optional[dict]:
    st = mp_io_stats() if io else None
    _check(lib.mp_merge_avg(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta), _ptr(mask),
                            _floats(alpha, len(experts)), _ptr(out), _io(st), _stream(stream)))
    return st.as_dict() if io else None


def mp_merge_avg_renorm(layout: Layout, base, experts, mask, alpha, out, residency: int = MP_DEVICE,
                        io: bool = False, stream=None, delta: bool = False) -> Optional[dict]:
    """Selected-only AVG: alpha renormalised over each block's selected experts."""
    st = mp_io_stats() if io else None
    _check(lib.mp_merge_avg_renorm(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta),
                                   _ptr(mask),
                                   _floats(alpha, len(experts)), _ptr(out), _io(st), _stream(stream)))
    return st.as_dict() if io else None


def mp_merge_ties(layout: Layout, base, experts, mask, density: float, lam: float, out,
                  residency: int = MP_DEVICE, io: bool = False, stream=None, delta: bool = False) -> Optional[dict]:
    st = mp_io_stats() if io else None
    _check(lib.mp_merge_ties(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta), _ptr(mask),
                             float(density), float(lam), _ptr(out), _io(st), _stream(stream)))
    return st.as_dict() if io else None


def mp_merge_ties_tau(layout: Layout, base, experts, mask, tau, lam: float, out, residency: int = MP_DEVICE,
                      io: bool = False, stream=None, delta: bool = False) -> Optional[dict]:
    st = mp_io_stats() if io else None
    _check(lib.mp_merge_ties_tau(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta),
                                 _ptr(mask),
                                 _ptr(tau), float(lam), _ptr(out), _io(st), _stream(stream)))
    return st.as_dict() if io else None


def mp_merge_dare(layout: Layout, base, experts, mask, p: float, seed: int, combine: int, alpha, lam: float,
                  out, residency: int = MP_DEVICE, io: bool = False, stream=None,
                  delta: bool = False) -> Optional[dict]:
    st = mp_io_stats() if io else None
    a = _floats(alpha, len(experts)) if alpha is not None else None
    _check(lib.mp_merge_dare(layout.ref, _ptr(base), _ptrs(experts), len(experts), _res(residency, delta), _ptr(mask),
                             float(p), int(seed) & 0xFFFFFFFF, int(combine), a, float(lam), _ptr(out), _io(st),
                             _stream(stream)))
    return st.as_dict() if io else None


def mp_lora_materialize(layout: Layout, loras, adapters, deltas, mask=None, stream=None):
    """Explicit-delta checkpoints drawn from LoRA adapters (selected units only).

    ``loras``: records (tensor, rows, cols, rank, a_off, b_off, scale);
    ``adapters``/``deltas``: K device tensors each (adapters may be empty
    when there are no records)."""
    recs = (mp_lora_tensor * max(len(loras), 1))(
        *[mp_lora_tensor(int(t), int(rank), int(rows), int(cols), int(a), int(b), float(sc))
          for (t, rows, cols, rank, a, b, sc) in loras])
    K = len(deltas)
    _check(lib.mp_lora_materialize(layout.ref, recs, len(loras), _ptrs(adapters) if loras else None, K, _ptr(mask),
                                   _ptrs(deltas), _stream(stream)))


def mp_lora_merge_ties_tau(layout: Layout, base, loras, adapters, mask, tau, lam, out, stream=None):
    """Budgeted TIES from catalog thresholds with every selected delta drawn
    from the adapters inside the merge (no delta checkpoint): equal to
    ``mp_lora_materialize(mask)`` then ``mp_merge_ties_tau(delta=True)``.

    ``loras`` as for mp_lora_materialize; ``adapters``: K device tensors
    (K entries of None when there are no records); ``mask``: device
    int32[G]; ``tau``: device int32[G*K]."""
    recs = (mp_lora_tensor * max(len(loras), 1))(
        *[mp_lora_tensor(int(t), int(rank), int(rows), int(cols), int(a), int(b), float(sc))
          for (t, rows, cols, rank, a, b, sc) in loras])
    K = len(adapters)
    _check(lib.mp_lora_merge_ties_tau(layout.ref, _ptr(base), recs, len(loras), _ptrs(adapters) if loras else None,
                                      K, _ptr(mask),
                                      _ptr(tau), float(lam), _ptr(out), _stream(stream)))


# ------------------------------------------------------------------ the feed-forward part of a block
@functools.lru_cache(maxsize=None)
def _code_of(dtype) -> int:
    import torch
    if dtype is torch.bfloat16:
        return MP_BF16
    if dtype is torch.float32:
        return MP_F32
    raise ValueError(f"dtype {dtype} is not torch.float32 or torch.bfloat16")


def _dtype_code(t) -> int:
    return _code_of(t.dtype)


def _matrix(t, rows, cols, dtype, name: str) -> int:
    """Checks a rows x cols matrix of unit column stride; its row stride."""
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(rows, cols)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    sr, sc = t.stride()
    if sc != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if rows > 1:
        if sr < cols:
            raise ValueError(f"{name}: rows overlap or run backwards (stride {sr})")
        return sr
    return max(sr, cols)


def _vector(t, n, dtype, name: str):
    if t is not None:
        if t.numel() != n or t.dtype is not dtype or not t.is_contiguous():
            raise ValueError(f"{name}: expected {n} contiguous values of {dtype}")


def _scratch(need: int, workspace, like, stream):
    """(pointer, bytes) of the caller's workspace tensor, or of a new one whose memory torch's allocator
    keeps for the call's stream; the tensor is returned to be held until the launch."""
    if need == 0:
        return None, 0, None
    import torch
    if workspace is None:
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
        else:
            if isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=like.device)
            with torch.cuda.stream(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    if not workspace.is_contiguous():
        raise ValueError("workspace: must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _linear_shape(dtype, act, m, n, k, ldx=0, ldw=0, ldy=0, ldz=0, ldr=0):
    return mp_linear_shape(dtype, int(act), m, n, k, ldx, ldw, ldy, ldz, ldr)


def _need(fn, *args) -> int:
    n = C.c_uint64(0)
    _check(fn(*args, C.byref(n)))
    return n.value


def mp_linear(x, w, y, bias=None, residual=None, act: int = MP_ACT_NONE, z=None, workspace=None, stream=None):
    """y = act(z) + residual with z = x w^T + bias, into `y` (and `z`, if given).

    ``x``: [m, k]; ``w``: [n, k], as checkpoints hold it; ``y``, ``z``, ``residual``: [m, n]; ``bias``: [n].
    fp32 or bf16 device tensors, any row stride; ``residual`` may be ``y``.  ``workspace``: a device
    tensor of ``mp_linear_workspace`` bytes to reuse between calls (default: a new one)."""
    dt = x.dtype
    m, k = x.shape
    n = w.shape[0]
    s = _linear_shape(_dtype_code(x), act, m, n, k, _matrix(x, m, k, dt, "x"), _matrix(w, n, k, dt, "w"),
                      _matrix(y, m, n, dt, "y"), 0 if z is None else _matrix(z, m, n, dt, "z"),
                      0 if residual is None else _matrix(residual, m, n, dt, "residual"))
    _vector(bias, n, dt, "bias")
    ref = C.byref(s)
    wp, wb, hold = _scratch(mp_linear_workspace(s.dtype, s.act, m, n, k), workspace, x, stream)
    _check(lib.mp_linear(ref, x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(residual), y.data_ptr(), _ptr(z), wp, wb,
                         _stream(stream)))


def mp_linear_backward(dy, x=None, w=None, z=None, act: int = MP_ACT_NONE, dx=None, dw=None, dbias=None,
                       workspace=None, stream=None):
    """Gradients of ``mp_linear`` into those of ``dx`` [m, k], ``dw`` [n, k] and ``dbias`` [n] that are given.

    ``dy``: [m, n]; ``z``: the pre-activations that mp_linear stored (needed with an activation); ``x`` is
    needed for dw, ``w`` for dx.  The residual's gradient is dy."""
    dt = dy.dtype
    m, n = dy.shape
    if (dx is None) != (dx is None or w is None) or (dw is None) != (dw is None or x is None):
        raise ValueError("dx needs w, and dw needs x")
    k = dx.shape[1] if dx is not None else dw.shape[1] if dw is not None else 0
    if act != MP_ACT_NONE and z is None:
        raise ValueError("an activation needs z")
    s = _linear_shape(_dtype_code(dy), act, m, n, k, 0 if dw is None else _matrix(x, m, k, dt, "x"),
                      0 if dx is None else _matrix(w, n, k, dt, "w"), _matrix(dy, m, n, dt, "dy"),
                      0 if act == MP_ACT_NONE else _matrix(z, m, n, dt, "z"))
    lddx = 0 if dx is None else _matrix(dx, m, k, dt, "dx")
    lddw = 0 if dw is None else _matrix(dw, n, k, dt, "dw")
    _vector(dbias, n, dt, "dbias")
    ref = C.byref(s)
    wp, wb, hold = _scratch(mp_linear_workspace(s.dtype, s.act, m, n, k, True), workspace, dy, stream)
    _check(lib.mp_linear_backward(ref, dy.data_ptr(), _ptr(x) if dw is not None else None,
                                  _ptr(w) if dx is not None else None, _ptr(z) if act != MP_ACT_NONE else None,
                                  _ptr(dx), lddx, _ptr(dw), lddw, _ptr(dbias), wp, wb, _stream(stream)))


@functools.lru_cache(maxsize=1024)
def mp_linear_workspace(dtype: int, act: int, m: int, n: int, k: int, backward: bool = False) -> int:
    s = _linear_shape(dtype, act, m, n, k)
    return _need(lib.mp_linear_workspace, C.byref(s), int(backward))


def mp_norm(x, y, weight=None, bias=None, eps: float = 1e-6, rms: bool = False, mean=None, rstd=None, stream=None):
    """Layer norm (``rms``: RMS norm) of the rows of ``x`` [rows, cols] into ``y``, which may be ``x``;
    per-row statistics into the fp32 ``mean`` and ``rstd`` [rows], if given."""
    dt = x.dtype
    rows, cols = x.shape
    s = mp_norm_shape(_dtype_code(x), MP_NORM_RMS if rms else 0, rows, cols, _matrix(x, rows, cols, dt, "x"),
                      _matrix(y, rows, cols, dt, "y"), eps)
    _vector(weight, cols, dt, "weight")
    _vector(bias, cols, dt, "bias")
    _stats(rows, mean, rstd)
    _check(lib.mp_norm(C.byref(s), x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), _ptr(mean), _ptr(rstd),
                       _stream(stream)))


def _stats(rows, *ts):
    import torch
    for t in ts:
        _vector(t, rows, torch.float32, "mean or rstd")


def mp_norm_backward(dy, x, rstd, mean=None, weight=None, rms: bool = False, dx=None, dweight=None, dbias=None,
                     workspace=None, stream=None):
    """Gradients of ``mp_norm`` into those of ``dx`` [rows, cols] (which may be ``dy``), ``dweight`` and
    ``dbias`` [cols] that are given, from the statistics that mp_norm stored."""
    dt = x.dtype
    rows, cols = x.shape
    s = mp_norm_shape(_dtype_code(x), MP_NORM_RMS if rms else 0, rows, cols, _matrix(x, rows, cols, dt, "x"),
                      _matrix(dy, rows, cols, dt, "dy"), 0.0)
    lddx = 0 if dx is None else _matrix(dx, rows, cols, dt, "dx")
    _vector(weight, cols, dt, "weight")
    _vector(dweight, cols, dt, "dweight")
    _vector(dbias, cols, dt, "dbias")
    _stats(rows, mean, rstd)
    if mean is None and not rms:
        raise ValueError("layer norm needs mean")
    ref = C.byref(s)
    wp, wb, hold = _scratch(mp_norm_workspace(s.dtype, rows, cols, rms), workspace, x, stream)
    _check(lib.mp_norm_backward(ref, dy.data_ptr(), x.data_ptr(), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dx), lddx,
                                _ptr(dweight), _ptr(dbias), wp, wb, _stream(stream)))


@functools.lru_cache(maxsize=1024)
def mp_norm_workspace(dtype: int, rows: int, cols: int, rms: bool = False) -> int:
    s = mp_norm_shape(dtype, MP_NORM_RMS if rms else 0, rows, cols, cols, cols, 0.0)
    return _need(lib.mp_norm_workspace, C.byref(s))


@dataclass
class MoeLayer:
    """mp_moe_layer: where an expert's checkpoint holds its feed-forward matrices (element offsets; gate and
    up are ffn x hidden, down is hidden x ffn; up_off None: no up matrix), and how tokens are routed."""

    hidden: int
    ffn: int
    top_k: int
    gate_off: int
    up_off: Optional[int]
    down_off: int
    act: int = MP_ACT_SILU
    renorm: bool = False

    def _struct(self, dtype: int):
        return mp_moe_layer(dtype, int(self.act), self.top_k, MP_MOE_RENORM if self.renorm else 0, self.hidden,
                            self.ffn, self.gate_off, -1 if self.up_off is None else self.up_off, self.down_off)


def mp_moe(layer: MoeLayer, x, router, experts, y, ids=None, gates=None, router_bias=None, residual=None,
           residency: int = MP_DEVICE, workspace=None, stream=None):
    """A mixture-of-experts layer for a few tokens: ``x`` [tokens, hidden] through the ``top_k`` experts that
    ``router`` [E, hidden] chooses, into ``y``; the choices into ``ids`` (int32) and ``gates`` (fp32)
    [tokens, top_k], if given.  ``experts``: E flat checkpoints (residency MP_DEVICE or MP_HOST_PINNED)."""
    import torch
    dt = x.dtype
    T, D = x.shape
    E = len(experts)
    s = layer._struct(_dtype_code(x))
    ldx, ldy = _matrix(x, T, layer.hidden, dt, "x"), _matrix(y, T, D, dt, "y")
    ldr = 0 if residual is None else _matrix(residual, T, D, dt, "residual")
    if router.shape != (E, D) or router.dtype is not dt or not router.is_contiguous():
        raise ValueError(f"router: expected a contiguous {(E, D)} matrix of {dt}")
    _vector(router_bias, E, dt, "router_bias")
    _vector(ids, T * layer.top_k, torch.int32, "ids")
    _vector(gates, T * layer.top_k, torch.float32, "gates")
    need = max(layer.gate_off, layer.down_off, layer.up_off or 0) + layer.hidden * layer.ffn
    for e in experts:
        if e.dtype is not dt or e.numel() < need or not e.is_contiguous():
            raise ValueError(f"experts: expected flat checkpoints of at least {need} values of {dt}")
    ref = C.byref(s)
    wp, wb, hold = _scratch(_need(lib.mp_moe_workspace, ref, T), workspace, x, stream)
    ptrs = (C.c_void_p * max(E, 1))(*[e.data_ptr() for e in experts])
    _check(lib.mp_moe(ref, T, x.data_ptr(), ldx, router.data_ptr(), _ptr(router_bias), ptrs, E, residency,
                      _ptr(residual), ldr, y.data_ptr(), ldy, _ptr(ids), _ptr(gates), wp, wb, _stream(stream)))


def mp_moe_workspace(layer: MoeLayer, dtype: int, tokens: int) -> int:
    s = layer._struct(dtype)
    return _need(lib.mp_moe_workspace, C.byref(s), tokens)


# ------------------------------------------------------------------ attention over a paged cache
@functools.lru_cache(maxsize=None)
def _ints():
    import torch
    return torch.int32, torch.int64, torch.float64


def _heads(t, shape, dtype, name: str):
    """Checks [tokens, heads, dim] values of unit stride inside a head; (token stride, head stride)."""
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    st, sh, sd = t.stride()
    if sd != 1 and shape[2] > 1:
        raise ValueError(f"{name}: the values of a head must be adjacent")
    return st, sh


def _head_rows(t, shape, dtype, name: str) -> int:
    """The same with the heads of a token side by side; its token stride."""
    tokens, heads, dim = shape
    if t.shape == shape and t.dtype is dtype:
        st, sh, sd = t.stride()
        if sd == 1 and sh == dim and tokens > 1:
            return st
    st, sh = _heads(t, shape, dtype, name)
    if sh != dim and heads > 1:
        raise ValueError(f"{name}: the heads of a token must be adjacent")
    return st if tokens > 1 else max(st, heads * dim)


def _turn_args(tokens, positions, freqs) -> int:
    """Checks them; the number of turned values of a head."""
    if freqs is None:
        return 0
    _, i64, f64 = _ints()
    pairs = freqs.numel()
    _vector(freqs, pairs, f64, "freqs")
    if positions is None:
        raise ValueError("freqs need positions")
    _vector(positions, tokens, i64, "positions")
    return 2 * pairs


def mp_rope_frequencies(rot_dim: int, base: float = 10000.0, kind: int = MP_ROPE_PLAIN, factor: float = 1.0,
                        original: float = 0.0, low: float = 1.0, high: float = 4.0):
    """(freqs, amplitude): the frequencies of a model's rotary positions, a float64 host tensor of rot_dim / 2 values
    (radians per position; the calls take it on the device), and the factor of the turned values.

    ``kind``: MP_ROPE_PLAIN, MP_ROPE_LINEAR, MP_ROPE_NTK, MP_ROPE_PARTS or MP_ROPE_YARN; ``factor``: of the context's
    extension; ``original``: tokens of the context before it, ``low`` and ``high``: turns in it below which a pair is
    slowed by the whole factor and above which it is kept."""
    import torch
    freqs = torch.empty(max(int(rot_dim), 0) // 2, dtype=torch.float64)
    amplitude = C.c_float(0)
    s = mp_rope_scaling(int(kind), base, factor, original, low, high)
    _check(lib.mp_rope_frequencies(C.byref(s), int(rot_dim), C.cast(freqs.data_ptr(), C.POINTER(C.c_double)),
                                   C.byref(amplitude)))
    return freqs, float(amplitude.value)


def _rope(call, x, y, names, positions, freqs, interleaved, amplitude, back, stream):
    dt, shape = x.dtype, x.shape
    T, H, D = shape
    sx, sy = _heads(x, shape, dt, names[0]), _heads(y, shape, dt, names[1])
    rot = _turn_args(T, positions, freqs)
    if back:
        sx, sy = sy, sx
    s = mp_rope_shape(_code_of(dt), MP_ROPE_INTERLEAVED if interleaved else 0, T, H, D, rot, *sx, *sy, amplitude)
    _check(call(C.byref(s), x.data_ptr(), _ptr(positions), _ptr(freqs), y.data_ptr(), _stream(stream)))


def mp_rope(x, y, positions, freqs, interleaved: bool = False, amplitude: float = 1.0, stream=None):
    """Rotary positions: the first 2 len(freqs) values of each head of ``x`` [tokens, heads, dim] turned by
    positions * freqs, the others copied, into ``y``, which may be ``x``.

    fp32 or bf16 device tensors of any token and head strides; ``positions``: int64 [tokens]; ``freqs``: float64
    (``mp_rope_frequencies``).  Pairs are (i, i + len(freqs)), or ``interleaved`` (2 i, 2 i + 1)."""
    _rope(lib.mp_rope, x, y, ("x", "y"), positions, freqs, interleaved, amplitude, False, stream)


def mp_rope_backward(dy, dx, positions, freqs, interleaved: bool = False, amplitude: float = 1.0, stream=None):
    """Gradient of ``mp_rope``: ``dy`` turned back into ``dx``, which may be ``dy``."""
    _rope(lib.mp_rope_backward, dy, dx, ("dy", "dx"), positions, freqs, interleaved, amplitude, True, stream)


class KvCache:
    """mp_kv_cache: keys and values [pages, page_size, heads, dim], device tensors of the same type and, but in
    dimensions of one place, strides in which the values of a head are adjacent; they may be transposed views (heads
    before a page's tokens) and parts of one array."""

    def __init__(self, k, v):
        shape, strides, dt = k.shape, k.stride(), k.dtype
        if len(shape) != 4 or shape != v.shape or dt is not v.dtype:
            raise ValueError(f"k {tuple(shape)} {dt}, v {tuple(v.shape)} {v.dtype}: expected two equal "
                             "[pages, page_size, heads, dim]")
        if strides != v.stride() and any(a != b for n, a, b in zip(shape, strides, v.stride()) if n > 1):
            raise ValueError("k and v need equal strides")
        if strides[3] != 1 and shape[3] > 1:
            raise ValueError("k and v: the values of a head must be adjacent")
        self.k, self.v = k, v
        self._shape, self._dtype = shape, dt
        self._s = mp_kv_cache(_code_of(dt), 0, *shape, *strides[:3], k.data_ptr(), v.data_ptr())
        self._ref = C.byref(self._s)


def mp_kv_append(cache: KvCache, k, v, slots, positions=None, freqs=None, q=None, q_out=None,
                 interleaved: bool = False, amplitude: float = 1.0, stream=None):
    """Stores new tokens' keys ``k``, turned as ``mp_rope`` turns them, and values ``v`` [tokens, heads, dim] in the
    cache at ``slots`` (int64 [tokens], page * page_size + place; outside the cache: not stored), and the tokens'
    queries ``q`` [tokens, q_heads, dim], turned, in ``q_out`` (default: in place).  Without ``freqs`` nothing is
    turned."""
    dt, shape, held = cache._dtype, k.shape, cache._shape
    T, heads = shape[0], shape[1:]
    if heads != held[2:]:
        raise ValueError(f"k: heads {tuple(heads)}, the cache's are {tuple(held[2:])}")
    ldk, ldv = _head_rows(k, shape, dt, "k"), _head_rows(v, shape, dt, "v")
    _vector(slots, T, _ints()[1], "slots")
    rot = _turn_args(T, positions, freqs)
    hq = ldq = ldqo = 0
    if q is None:
        q_out = None
    else:
        hq = q.shape[1]
        shape = (T, hq, heads[1])
        ldq = ldqo = _head_rows(q, shape, dt, "q")
        if q_out is None:
            q_out = q
        else:
            ldqo = _head_rows(q_out, shape, dt, "q_out")
    r = mp_kv_rows(T, hq, rot, MP_ROPE_INTERLEAVED if interleaved else 0, amplitude, ldk, ldv, ldq, ldqo)
    _check(lib.mp_kv_append(cache._ref, C.byref(r), k.data_ptr(), v.data_ptr(), slots.data_ptr(),
                            positions.data_ptr() if rot else None, _ptr(freqs), _ptr(q), _ptr(q_out),
                            _stream(stream)))


def mp_kv_attend(cache: KvCache, q, table, lens, out, scale: Optional[float] = None, window: int = 0, lse=None,
                 workspace=None, stream=None):
    """Attention of one new token per row over the cache: ``q`` and ``out`` [rows, q_heads, dim] (``out`` may be
    ``q``), ``table`` int32 [rows, width], the pages of each row's sequence (an expanded row is taken), ``lens`` int32
    [rows], its length with the new token, whose key has been appended.

    ``scale``: of the scores, default dim^-0.5; ``window``: keys to look back, the token's own among them (0: all);
    ``lse``: fp32 [rows, q_heads], receives the log of the summed exponentials; ``workspace``: a device tensor of
    ``mp_kv_attend_workspace`` bytes to reuse between calls (default: a new one)."""
    i32 = _ints()[0]
    dt, D = cache._dtype, cache._shape[3]
    R, H = q.shape[:2]
    shape = (R, H, D)
    ldq, ldo = _head_rows(q, shape, dt, "q"), _head_rows(out, shape, dt, "out")
    wide = table.shape
    if len(wide) != 2 or wide[0] != R or table.dtype is not i32:
        raise ValueError(f"table: shape {tuple(wide)} {table.dtype}, expected int32 of {R} rows")
    W = wide[1]
    st, sc = table.stride()
    if W > 1 and sc != 1:
        raise ValueError("table: the pages of a row must be adjacent")
    if R > 1 and st != 0 and st < W:
        raise ValueError(f"table: rows overlap or run backwards (stride {st})")
    _vector(lens, R, i32, "lens")
    if lse is not None:
        import torch
        if lse.shape != (R, H):
            raise ValueError(f"lse: shape {tuple(lse.shape)}, expected {(R, H)}")
        _vector(lse, R * H, torch.float32, "lse")
    s = mp_kv_attend_shape(R, H, W, ldq, ldo, st if R > 1 else max(st, W), int(window),
                           D ** -0.5 if scale is None else scale)
    wp, wb, hold = _scratch(_kv_need(cache, s), workspace, q, stream)
    _check(lib.mp_kv_attend(cache._ref, C.byref(s), q.data_ptr(), table.data_ptr(), lens.data_ptr(), out.data_ptr(),
                            _ptr(lse), wp, wb, _stream(stream)))


def _kv_need(cache: KvCache, s) -> int:
    return _need(lib.mp_kv_attend_workspace, cache._ref, C.byref(s))


def mp_kv_attend_workspace(cache: KvCache, rows: int, q_heads: int, width: int, window: int = 0) -> int:
    """Workspace bytes of ``mp_kv_attend`` for a table of rows x width pages."""
    return _kv_need(cache, mp_kv_attend_shape(rows, q_heads, width, 0, 0, 0, window, 1.0))


def mp_last_error() -> str:
    return lib.mp_last_error().decode()


def mp_stream_copy(src, dst, stream=None):
    """Plain stream copy of src's bytes into dst (device tensors of equal
    byte size, a multiple of 16): a measurement aid for the HBM rate."""
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != n:
        raise ValueError("src and dst differ in size")
    _check(lib.mp_stream_copy(_ptr(src), _ptr(dst), n, _stream(stream)))


def mp_set_stage_bytes(nbytes: int):
    _check(lib.mp_set_stage_bytes(int(nbytes)))


def mp_set_workspace_limit(nbytes: int):
    """Cap on the library's cached workspace in bytes (0: none)."""
    _check(lib.mp_set_workspace_limit(int(nbytes)))


def mp_workspace_bytes() -> int:
    return int(lib.mp_workspace_bytes())


def mp_ties_tensor_left() -> int:
    """Pairs that the last ``mp_ties_tensor_thresholds`` call left to the digit
    passes (-1: it took every pair by those)."""
    return int(lib.mp_ties_tensor_left())


def mp_release():
    lib.mp_release()
