"""Thin ctypes binding over libretrace (the C ABI in include/retrace.h).

Argument marshalling only: every step of the round runs in the library's CUDA
kernels.  Tensors are torch CUDA tensors used as device buffers; the functions
carry the C entry points' names.  If the library has not been built the
import fails loudly -- there is no fallback path.
"""

from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

RETRACE_F32 = 0
RETRACE_BF16 = 1

_STATUS = {
    0: "RETRACE_OK",
    1: "RETRACE_ERR_INVALID_ARG",
    2: "RETRACE_ERR_UNSUPPORTED",
    3: "RETRACE_ERR_WORKSPACE",
    4: "RETRACE_ERR_CUDA",
    5: "RETRACE_ERR_DEVICE",
}


class RetraceError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def _load() -> ctypes.CDLL:
    path = _build.LIB_PATH
    if not os.path.exists(path):
        raise ImportError(
            f"libretrace.so is not built ({path}); run `python -m paper_2608_29748_gb300.build` "
            "or __graft_entry__.build() first"
        )
    lib = ctypes.CDLL(path)
    P, I, I64, SZ, F = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    lib.retrace_last_error.restype = ctypes.c_char_p
    lib.retrace_version.restype = ctypes.c_char_p
    lib.retrace_workspace_bytes.argtypes = [I, I, I, I, I]
    lib.retrace_workspace_bytes.restype = SZ
    lib.retrace_workspace_init.argtypes = [P, SZ, P]
    lib.retrace_workspace_check.argtypes = [P, SZ, ctypes.POINTER(ctypes.c_uint32), P]
    lib.retrace_verify.argtypes = [P, I, I, I, I, I64, I64, P, P, P, P, P, P, SZ, P]
    lib.retrace_align_refine.argtypes = [P, P, I, I, I, I, P, P, F, P, P, P, SZ, P]
    lib.retrace_gate_fuse.argtypes = [P, I64, I64, P, P, P, P, I, I, I, I, P, P, SZ, P]
    lib.retrace_round.argtypes = [P, I64, I64, P, P, P, P, I64, I64, P, P, P, F, I, I, I, I, I,
                                  P, P, P, P, P, P, P, SZ, ctypes.c_uint32, P, P]
    lib.retrace_round_lowrank.argtypes = [P, I64, I64, P, P, P, P, P, P, P, P, P, F, I, I, I, I, I,
                                          P, P, P, P, P, P, P, SZ, P, P]
    lib.retrace_verify_sampled.argtypes = [P, I64, I64, P, I64, I64, I, I, I, I, P, P, F, I, F, P, P, P, P, SZ, P]
    lib.retrace_wait_selftest.argtypes = [I, P, ctypes.c_uint32, P, SZ, P]
    lib.retrace_set_verify_schedule.argtypes = [I]
    lib.retrace_verify_plan.argtypes = [I, I, I, I, I, ctypes.POINTER(ctypes.c_int)]
    lib.retrace_round_sampled.argtypes = [P, I64, I64, P, I64, I64, P, P, F, I, F, P, P, P, I64, I64, P, P, P, F,
                                          I, I, I, I, I, P, P, P, P, P, P, SZ, P, P]
    lib.retrace_kv_append.argtypes = [P, I64, I64, I, P, I64, I64, P, I64, I64, P, P, I, I, P, I, I, I, P, P, I64, I64, P]
    lib.retrace_attend_workspace_bytes.argtypes = [I, I, I, I]
    lib.retrace_attend_workspace_bytes.restype = SZ
    lib.retrace_attend.argtypes = [P, I64, I64, I, P, P, I, I, F, I, I, I, P, P, I64, I64, P, SZ, P]
    lib.retrace_sample.argtypes = [P, I, I, I, I, I64, I64, P, P, P, P, P, P, P, P]
    for name in ("retrace_kv_append", "retrace_attend", "retrace_sample",
                 "retrace_workspace_init", "retrace_workspace_check", "retrace_verify",
                 "retrace_align_refine", "retrace_gate_fuse", "retrace_round", "retrace_round_lowrank",
                 "retrace_verify_sampled", "retrace_round_sampled", "retrace_wait_selftest",
                 "retrace_set_verify_schedule", "retrace_verify_plan"):
        getattr(lib, name).restype = I
    return lib


lib = _load()


def _check(status: int) -> None:
    if status != 0:
        raise RetraceError(status, lib.retrace_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return RETRACE_BF16
    if t.dtype == torch.float32:
        return RETRACE_F32
    raise TypeError(f"unsupported floating dtype {t.dtype}")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libretrace takes CUDA tensors")
    return t.data_ptr()


# The current stream's handle without building a torch Stream object (0.1
# against 3 us of a call that takes 10 to 20 us to enqueue).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _current_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def retrace_workspace_bytes(B: int, K: int, V: int, d: int, dtype: torch.dtype) -> int:
    code = RETRACE_BF16 if dtype == torch.bfloat16 else RETRACE_F32
    return int(lib.retrace_workspace_bytes(B, K, V, d, code))


class Workspace:
    """Caller-owned device workspace sized for (B, K, V, d, dtype), zeroed once."""

    def __init__(self, B, K, V, d, dtype, device=None, stream=None):
        self._allocate(retrace_workspace_bytes(B, K, V, d, dtype), device, stream)

    def _allocate(self, nbytes, device, stream):
        self.nbytes = nbytes
        if self.nbytes == 0:
            raise ValueError("invalid workspace shape")
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device or "cuda")
        base = self.buf.data_ptr()
        self.ptr = (base + 255) // 256 * 256
        retrace_workspace_init(self, stream)

    def check(self, stream=None) -> int:
        return retrace_workspace_check(self, stream)


def retrace_workspace_init(ws: Workspace, stream=None) -> None:
    _check(lib.retrace_workspace_init(ws.ptr, ws.nbytes, _stream(stream)))


def retrace_workspace_check(ws: Workspace, stream=None) -> int:
    flags = ctypes.c_uint32(0)
    st = lib.retrace_workspace_check(ws.ptr, ws.nbytes, ctypes.byref(flags), _stream(stream))
    if st not in (0, 5):
        _check(st)
    return int(flags.value)


def _int32(t: torch.Tensor, name: str) -> None:
    if t.dtype != torch.int32:
        raise TypeError(f"{name} must be int32")


def retrace_verify(logits, draft, accept_len, committed, bonus, ws, target_argmax=None, stream=None):
    """Greedy verification (see include/retrace.h).  logits [B, K+1, V], last dim contiguous."""
    B, K1, V = logits.shape
    if logits.stride(2) != 1:
        raise ValueError("logits: vocabulary dimension must be contiguous")
    for t, n in ((draft, "draft"), (accept_len, "accept_len"), (committed, "committed"), (bonus, "bonus")):
        _int32(t, n)
    _check(lib.retrace_verify(_ptr(logits), _dtype_code(logits), B, K1 - 1, V, logits.stride(1),
                              logits.stride(0), _ptr(draft), _ptr(accept_len), _ptr(committed),
                              _ptr(bonus), _ptr(target_argmax), ws.ptr, ws.nbytes, _stream(stream)))


def retrace_align_refine(hD, hT, accept_len, Wc, beta, r_out, n_out, ws, stream=None):
    """Alignment + target-aware correction: r_out [B, K, d], n_out [B]."""
    B, K, d = hD.shape
    for t in (hD, hT, Wc, r_out):
        if not t.is_contiguous():
            raise ValueError("hD, hT, Wc and r_out must be contiguous")
    _check(lib.retrace_align_refine(_ptr(hD), _ptr(hT), _dtype_code(hD), B, K, d, _ptr(accept_len),
                                    _ptr(Wc), float(beta), _ptr(r_out), _ptr(n_out), ws.ptr,
                                    ws.nbytes, _stream(stream)))


def _e_strides(e: torch.Tensor, B: int, K: int, d: int):
    if e.dim() == 1:
        return 0, 0
    if e.shape != (B, K, d) or not e.is_contiguous():
        raise ValueError("e must be a [d] vector or a contiguous [B, K, d] tensor")
    return K * d, d


def retrace_gate_fuse(e, r, n, Wv, Wg, e_out, ws, stream=None):
    """Gated residual conditioning: e_out [B, K, d]."""
    B, K, d = r.shape
    ebs, eps = _e_strides(e, B, K, d)
    _check(lib.retrace_gate_fuse(_ptr(e), ebs, eps, _ptr(r), _ptr(n), _ptr(Wv), _ptr(Wg),
                                 _dtype_code(r), B, K, d, _ptr(e_out), ws.ptr, ws.nbytes,
                                 _stream(stream)))


# retrace_round flags (include/retrace.h)
ROUND_OVERLAP = 0x1
COND_RAW = 0x2
COND_OVERWRITE = 0x4
COND_NONE = 0x8


def retrace_round(logits, draft, hD, hT, e, Wc, Wv, Wg, beta, accept_len, committed, bonus, e_out,
                  ws, n_out=None, target_argmax=None, flags=0, phase_events=None, stream=None):
    """One round on one stream (see include/retrace.h); `flags` selects the
    overlapped kernel or an ablation variant."""
    B, K1, V = logits.shape
    K = K1 - 1
    d = hD.shape[2]
    if logits.stride(2) != 1:
        raise ValueError("logits: vocabulary dimension must be contiguous")
    ebs, eps = _e_strides(e, B, K, d)
    ev = None
    if phase_events is not None:
        ev = (ctypes.c_void_p * 4)(*[x._as_parameter_.value for x in phase_events])
    _check(lib.retrace_round(_ptr(logits), logits.stride(1), logits.stride(0), _ptr(draft), _ptr(hD),
                             _ptr(hT), _ptr(e), ebs, eps, _ptr(Wc), _ptr(Wv), _ptr(Wg), float(beta),
                             _dtype_code(logits), B, K, V, d, _ptr(accept_len), _ptr(committed),
                             _ptr(bonus), _ptr(target_argmax), _ptr(n_out), _ptr(e_out), ws.ptr,
                             ws.nbytes, int(flags),
                             ctypes.cast(ev, ctypes.c_void_p) if ev is not None else None,
                             _stream(stream)))


def retrace_verify_sampled(target_logits, draft_logits, draft, uniforms, temperature, top_k, top_p, accept_len,
                           committed, bonus, ws, stream=None):
    """Speculative sampling of one block per sequence (see include/retrace.h)."""
    _check_sampled(target_logits, draft_logits, uniforms)
    B, K1, V = target_logits.shape
    K = K1 - 1
    for t, name in ((draft, "draft"), (accept_len, "accept_len"), (committed, "committed"), (bonus, "bonus")):
        _int32(t, name)
    _check(lib.retrace_verify_sampled(_ptr(target_logits), target_logits.stride(1), target_logits.stride(0),
                                      _ptr(draft_logits), draft_logits.stride(1), draft_logits.stride(0),
                                      _dtype_code(target_logits), B, K, V, _ptr(draft), _ptr(uniforms),
                                      float(temperature), int(top_k), float(top_p), _ptr(accept_len),
                                      _ptr(committed), _ptr(bonus), ws.ptr, ws.nbytes, _stream(stream)))


def _check_sampled(target_logits, draft_logits, uniforms):
    B, K1, V = target_logits.shape
    K = K1 - 1
    if target_logits.stride(2) != 1 or draft_logits.stride(2) != 1:
        raise ValueError("logits: vocabulary dimension must be contiguous")
    if tuple(draft_logits.shape) != (B, K, V) or draft_logits.dtype != target_logits.dtype:
        raise ValueError("draft_logits must be [B, K, V] of the target logits' dtype")
    if uniforms.dtype != torch.float32 or tuple(uniforms.shape) != (B, K1) or not uniforms.is_contiguous():
        raise ValueError("uniforms must be contiguous float32 [B, K+1]")


def retrace_round_sampled(target_logits, draft_logits, draft, uniforms, temperature, top_k, top_p, hD, hT, e, Wc,
                          Wv, Wg, beta, accept_len, committed, bonus, e_out, ws, n_out=None, phase_events=None,
                          stream=None):
    """One round with sampled verification (see include/retrace.h)."""
    _check_sampled(target_logits, draft_logits, uniforms)
    B, K1, V = target_logits.shape
    K = K1 - 1
    d = hD.shape[2]
    for t, name in ((draft, "draft"), (accept_len, "accept_len"), (committed, "committed"), (bonus, "bonus")):
        _int32(t, name)
    ebs, eps = _e_strides(e, B, K, d)
    ev = None
    if phase_events is not None:
        ev = (ctypes.c_void_p * 4)(*[x._as_parameter_.value for x in phase_events])
    _check(lib.retrace_round_sampled(_ptr(target_logits), target_logits.stride(1), target_logits.stride(0),
                                     _ptr(draft_logits), draft_logits.stride(1), draft_logits.stride(0), _ptr(draft),
                                     _ptr(uniforms), float(temperature), int(top_k), float(top_p), _ptr(hD), _ptr(hT),
                                     _ptr(e), ebs, eps, _ptr(Wc), _ptr(Wv), _ptr(Wg), float(beta),
                                     _dtype_code(target_logits), B, K, V, d, _ptr(accept_len), _ptr(committed),
                                     _ptr(bonus), _ptr(n_out), _ptr(e_out), ws.ptr, ws.nbytes,
                                     ctypes.cast(ev, ctypes.c_void_p) if ev is not None else None,
                                     _stream(stream)))


def retrace_round_lowrank(logits, draft, hD, hT, e, P, Bc, Ac, Wv, Wg, beta, accept_len, committed, bonus,
                          e_out, ws, n_out=None, target_argmax=None, phase_events=None, stream=None):
    """One round with the low-rank conditioning path (see include/retrace.h)."""
    B, K1, V = logits.shape
    K = K1 - 1
    d = hD.shape[2]
    if logits.stride(2) != 1:
        raise ValueError("logits: vocabulary dimension must be contiguous")
    if e.dim() != 1:
        raise ValueError("e: the low-rank path takes one broadcast vector [d]")
    ev = None
    if phase_events is not None:
        ev = (ctypes.c_void_p * 4)(*[x._as_parameter_.value for x in phase_events])
    _check(lib.retrace_round_lowrank(_ptr(logits), logits.stride(1), logits.stride(0), _ptr(draft), _ptr(hD),
                                     _ptr(hT), _ptr(e), _ptr(P), _ptr(Bc), _ptr(Ac), _ptr(Wv), _ptr(Wg),
                                     float(beta), _dtype_code(logits), B, K, V, d, _ptr(accept_len),
                                     _ptr(committed), _ptr(bonus), _ptr(target_argmax), _ptr(n_out), _ptr(e_out),
                                     ws.ptr, ws.nbytes,
                                     ctypes.cast(ev, ctypes.c_void_p) if ev is not None else None,
                                     _stream(stream)))


def retrace_wait_selftest(kind, flag, target, ws, stream=None):
    """Runs the kernels' bounded wait on a caller-controlled condition (see include/retrace.h)."""
    if flag is not None and flag.dtype != torch.int32:
        raise TypeError("flag must be an int32 device tensor")
    _check(lib.retrace_wait_selftest(int(kind), _ptr(flag), int(target), ws.ptr, ws.nbytes, _stream(stream)))


class RoundBuffers:
    """Device outputs of one round for a (B, K, d) shape."""

    def __init__(self, B, K, d, dtype, device="cuda"):
        self.accept_len = torch.empty(B, dtype=torch.int32, device=device)
        self.committed = torch.empty(B, K + 1, dtype=torch.int32, device=device)
        self.bonus = torch.empty(B, dtype=torch.int32, device=device)
        self.n = torch.empty(B, dtype=torch.int32, device=device)
        self.e_out = torch.empty(B, K, d, dtype=dtype, device=device)


def run_round(x: dict, ws: Workspace, out: RoundBuffers | None = None, target_argmax=None,
              flags=0, phase_events=None, stream=None) -> RoundBuffers:
    """retrace_round over a dict of device tensors (keys as in workloads.make_round_inputs)."""
    logits = x["logits"]
    B, K1, _ = logits.shape
    d = x["hD"].shape[2]
    if out is None:
        out = RoundBuffers(B, K1 - 1, d, logits.dtype, logits.device)
    retrace_round(logits, x["draft"], x["hD"], x["hT"], x["e"], x["Wc"], x["Wv"], x["Wg"], x["beta"],
                  out.accept_len, out.committed, out.bonus, out.e_out, ws, n_out=out.n,
                  target_argmax=target_argmax, flags=flags, phase_events=phase_events, stream=stream)
    return out


def version() -> str:
    return lib.retrace_version().decode()


VERIFY_AUTO, VERIFY_FULL, VERIFY_WINDOWS = 0, 1, 2


def retrace_verify_plan(B: int, K: int, V: int, dtype: torch.dtype, target_argmax: bool = False) -> list[int]:
    """Window boundaries greedy verification takes for this shape under the
    current schedule ([0, K+1] for the one-pass schedule)."""
    starts = (ctypes.c_int * 17)()
    code = RETRACE_BF16 if dtype == torch.bfloat16 else RETRACE_F32 if dtype == torch.float32 else -1
    n = lib.retrace_verify_plan(B, K, V, code, int(bool(target_argmax)), starts)
    if n < 1:
        raise RetraceError(1, "invalid shape or dtype for retrace_verify_plan")
    return list(starts[: n + 1])


def retrace_set_verify_schedule(mode: int) -> int:
    """Selects the greedy verification schedule (VERIFY_AUTO / VERIFY_FULL /
    VERIFY_WINDOWS); returns the previous one."""
    prev = lib.retrace_set_verify_schedule(int(mode))
    if prev < 0:
        raise RetraceError(1, f"unknown verification schedule {mode}")
    return prev


def run_round_lowrank(x: dict, w: dict, ws: Workspace, out: RoundBuffers | None = None, target_argmax=None,
                      phase_events=None, stream=None) -> RoundBuffers:
    """retrace_round_lowrank over the round inputs ``x`` and low-rank weights ``w``
    (keys as in workloads.make_round_inputs / make_lowrank_weights)."""
    logits = x["logits"]
    B, K1, _ = logits.shape
    d = x["hD"].shape[2]
    if out is None:
        out = RoundBuffers(B, K1 - 1, d, logits.dtype, logits.device)
    retrace_round_lowrank(logits, x["draft"], x["hD"], x["hT"], x["e"], w["P"], w["Bc"], w["Ac"], w["Wv_lr"],
                          w["Wg_lr"], x["beta"], out.accept_len, out.committed, out.bonus, out.e_out, ws,
                          n_out=out.n, target_argmax=target_argmax, phase_events=phase_events, stream=stream)
    return out


def run_round_sampled(x: dict, s: dict, ws: Workspace, out: RoundBuffers | None = None, phase_events=None,
                      stream=None) -> RoundBuffers:
    """retrace_round_sampled over the round inputs ``x`` (its logits are the
    target's) and the sampling inputs ``s`` (keys as in
    workloads.make_sampled_inputs; its draft tokens replace x["draft"])."""
    logits = x["logits"]
    B, K1, _ = logits.shape
    d = x["hD"].shape[2]
    if out is None:
        out = RoundBuffers(B, K1 - 1, d, logits.dtype, logits.device)
    retrace_round_sampled(logits, s["draft_logits"], s["draft"], s["uniforms"], s["temperature"], s["top_k"],
                          s["top_p"], x["hD"], x["hT"], x["e"], x["Wc"], x["Wv"], x["Wg"], x["beta"], out.accept_len,
                          out.committed, out.bonus, out.e_out, ws, n_out=out.n, phase_events=phase_events,
                          stream=stream)
    return out


# ---- around the round: paged cache, attention over it, sampling ---------------

_FAR = 2**31 - 1
_append, _attend, _sample = lib.retrace_kv_append, lib.retrace_attend, lib.retrace_sample


class _KvCacheStruct(ctypes.Structure):  # retrace_kv_cache (include/retrace.h)
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("slot_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("num_pages", ctypes.c_int),
                ("page_size", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("max_pages", ctypes.c_int),
                ("dtype", ctypes.c_int)]


class KvCache:
    """A paged cache: k and v [num_pages, page_size, kv_heads, head_dim] (any strides,
    the same for both, head_dim contiguous) and page_table [B, max_pages] int32, whose rows are
    apart in memory (sequences may have the same pages).  Keeps the tensors; their contents may
    change between calls."""

    def __init__(self, k, v, page_table):
        if k.dim() != 4 or v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype or k.stride(3) != 1:
            raise ValueError("k and v must be [pages, page_size, kv_heads, head_dim] of one dtype and layout, head_dim contiguous")
        _int32(page_table, "page_table")
        if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be [B, max_pages], the pages of a sequence contiguous")
        # a row of the table begins where the one before has ended (the stride of one row is not used)
        if page_table.shape[0] > 1 and page_table.stride(0) < page_table.shape[1]:
            raise ValueError("the rows of page_table must not share storage: an expanded table needs .contiguous()")
        self.k, self.v, self.page_table = k, v, page_table
        self.B, self.kv_heads, self.head_dim, self.dtype = page_table.shape[0], k.shape[2], k.shape[3], k.dtype
        self.struct = _KvCacheStruct(_ptr(k), _ptr(v), k.stride(0), k.stride(1), k.stride(2), k.shape[0], k.shape[1],
                                     k.shape[2], k.shape[3], _ptr(page_table), max(page_table.stride(0), page_table.shape[1]),
                                     page_table.shape[1], _dtype_code(k))
        self.ref = ctypes.addressof(self.struct)
        self.scale = self.head_dim**-0.5
        self.shape_B, self.shape_B1, self.shape_token = (self.B,), (self.B + 1,), (self.kv_heads, self.head_dim)


# The checks below run on every call of a decoding loop whose kernels take a few
# microseconds, so each is one comparison on the way that is taken, and what
# exactly is wrong is worked out after one of them fails.
def _refuse_packed(cache, T, tensors):
    for name, t, heads in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("libretrace takes CUDA tensors")
        if t.dim() != 3 or t.shape[0] != T or t.shape[2] != cache.head_dim or t.dtype != cache.dtype or \
                (heads is not None and t.shape[1] != heads):
            raise ValueError(f"{name} must be [{T}, {heads or 'heads'}, {cache.head_dim}] of the cache's dtype")
        if t.stride(2) != 1:
            raise ValueError(f"{name}: head_dim must be contiguous")


def _refuse_lengths(cache, cache_len, q_start):
    for name, t, n in (("cache_len", cache_len, cache.B), ("q_start", q_start, cache.B + 1)):
        if t is None and name == "q_start":
            continue
        _int32(t, name)
        if not t.is_cuda:
            raise ValueError("libretrace takes CUDA tensors")
        if t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous [{n}]: the page table has {cache.B} rows")


def _lengths(cache, cache_len, q_start):
    """Device pointers of the lengths and of the list of starts."""
    if cache_len.dtype != torch.int32 or cache_len.shape != cache.shape_B or not cache_len.is_cuda or not cache_len.is_contiguous():
        _refuse_lengths(cache, cache_len, None)
    if q_start is None:
        return cache_len.data_ptr(), None
    if q_start.dtype != torch.int32 or q_start.shape != cache.shape_B1 or not q_start.is_cuda or not q_start.is_contiguous():
        _refuse_lengths(cache, cache_len, q_start)
    return cache_len.data_ptr(), q_start.data_ptr()


def retrace_kv_append(q, k, v, cache: KvCache, cache_len, rope, q_out=None, q_start=None, interleaved=False, stream=None):
    """Appends k and v [T, kv_heads, head_dim] to the cache, rotating k and q [T, q_heads, head_dim]
    (optional, into q_out) by rope [positions, rot/2, 2] (None: no rotation) on the way (see
    include/retrace.h)."""
    shape = k.shape
    T, dtype = shape[0], cache.dtype
    k_token, k_head, k_last = k.stride()
    v_token, v_head, v_last = v.stride()
    if shape[1:] != cache.shape_token or v.shape != shape or k.dtype != dtype or v.dtype != dtype or k_last != 1 or v_last != 1 or \
            not (k.is_cuda and v.is_cuda):
        _refuse_packed(cache, T, (("k", k, cache.kv_heads), ("v", v, cache.kv_heads)))
    q_ptr = out_ptr = None
    q_heads = q_token = q_head = o_token = o_head = 0
    if q is not None:
        if q_out is None:
            raise ValueError("q needs q_out, which may be q itself")
        shape = q.shape
        q_token, q_head, q_last = q.stride()
        o_token, o_head, o_last = q_out.stride()
        if shape[0] != T or shape[2] != cache.head_dim or q_out.shape != shape or q.dtype != dtype or q_out.dtype != dtype or \
                q_last != 1 or o_last != 1 or not (q.is_cuda and q_out.is_cuda):
            _refuse_packed(cache, T, (("q", q, None), ("q_out", q_out, q.shape[1])))
        q_heads, q_ptr, out_ptr = shape[1], q.data_ptr(), q_out.data_ptr()
    positions = rot = 0
    rope_ptr = None
    if rope is not None:
        if rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[2] != 2 or not rope.is_contiguous() or not rope.is_cuda:
            raise ValueError("rope must be a contiguous float32 [positions, rot/2, 2] on the GPU")
        positions, half, _ = rope.shape
        rot, rope_ptr = 2 * half, rope.data_ptr()
    len_ptr, start_ptr = _lengths(cache, cache_len, q_start)
    status = _append(q_ptr, q_token, q_head, q_heads, k.data_ptr(), k_token, k_head, v.data_ptr(), v_token, v_head, start_ptr, len_ptr,
                     cache.B, T, rope_ptr, positions, rot, interleaved, cache.ref, out_ptr, o_token, o_head, _stream(stream))
    if status:
        _check(status)


class AttendWorkspace(Workspace):
    """Workspace of retrace_attend: one serves every call of these head counts and size."""

    def __init__(self, q_heads, kv_heads, head_dim, dtype, device=None, stream=None):
        code = RETRACE_BF16 if dtype == torch.bfloat16 else RETRACE_F32
        self._allocate(int(lib.retrace_attend_workspace_bytes(q_heads, kv_heads, head_dim, code)), device, stream)


def retrace_attend(q, cache: KvCache, cache_len, out, ws: AttendWorkspace, q_start=None, scale=None, window=0, sinks=0,
                   causal=True, stream=None):
    """Attention of q [T, q_heads, head_dim] over the cache into out (see include/retrace.h);
    scale defaults to head_dim ** -0.5."""
    shape = q.shape
    q_token, q_head, q_last = q.stride()
    o_token, o_head, o_last = out.stride()
    if shape[2] != cache.head_dim or out.shape != shape or q.dtype != cache.dtype or out.dtype != cache.dtype or q_last != 1 or \
            o_last != 1 or not (q.is_cuda and out.is_cuda):
        _refuse_packed(cache, shape[0], (("q", q, None), ("out", out, shape[1])))
    len_ptr, start_ptr = _lengths(cache, cache_len, q_start)
    if not (0 <= window <= _FAR and 0 <= sinks <= _FAR):  # past 32 bits another number would arrive
        window, sinks = max(-1, min(window, _FAR)), max(-1, min(sinks, _FAR))
    status = _attend(q.data_ptr(), q_token, q_head, shape[1], start_ptr, len_ptr, cache.B, shape[0],
                     cache.scale if scale is None else scale, window, sinks, causal, cache.ref, out.data_ptr(), o_token, o_head,
                     ws.ptr, ws.nbytes, _stream(stream))
    if status:
        _check(status)


def _setting(t, shape, dtype, name):
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} {dtype} on the GPU")
    return t.data_ptr()


def retrace_sample(logits, uniforms, tokens, probs=None, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    """Draws tokens [B, R] from logits [B, R, V] with the settings of each sequence ([B]) and the
    given uniforms [B, R] (see include/retrace.h)."""
    B, R, V = logits.shape
    batch, step, last = logits.stride()
    if last != 1:
        raise ValueError("logits: vocabulary dimension must be contiguous")
    rows, each, f32, i32 = (B, R), (B,), torch.float32, torch.int32
    status = _sample(_ptr(logits), _dtype_code(logits), B, R, V, step, batch, _setting(uniforms, rows, f32, "uniforms"),
                     _setting(temperature, each, f32, "temperature"), _setting(top_k, each, i32, "top_k"),
                     _setting(top_p, each, f32, "top_p"), _setting(min_p, each, f32, "min_p"),
                     _setting(tokens, rows, i32, "tokens"), _setting(probs, rows, f32, "probs"), _stream(stream))
    if status:
        _check(status)
