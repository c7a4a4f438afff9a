"""ctypes binding of libclusterattn.so: argument marshalling only.

The functions mirror the C entry points (`cluster_qk`, `select_blocks`,
`cluster_attention_fwd`).  torch provides device memory and streams; every
step of the computation runs inside the library's CUDA kernels.  There is no
CPU fallback: if the library is missing or no CUDA device is present the calls
raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libclusterattn.so")

CA_OK = 0
CA_ERR_INVALID_ARG, CA_ERR_UNSUPPORTED, CA_ERR_WORKSPACE, CA_ERR_CUDA, CA_ERR_TIMEOUT = 1, 2, 3, 4, 5
CA_ERR_BAD_INDEX = 6
ERRORS = {1: "CA_ERR_INVALID_ARG", 2: "CA_ERR_UNSUPPORTED", 3: "CA_ERR_WORKSPACE", 4: "CA_ERR_CUDA",
          5: "CA_ERR_TIMEOUT", 6: "CA_ERR_BAD_INDEX"}
CA_DTYPE_FP32, CA_DTYPE_BF16 = 0, 1
CA_Y_IN, CA_ATTN_FP32, CA_QUERY_UNNORMALIZED, CA_METRIC_IN, CA_ATTN_FP8_QK = 1, 2, 4, 8, 16

EXPORTS = ("ca_workspace_bytes", "cluster_qk", "select_blocks", "cluster_attention_fwd",
           "ca_last_status", "ca_attn_recomputed", "ca_version", "ca_kernel_launches", "cluster_attention_fwd_static",
           "ca_static_scratch_bytes", "ca_static_last_status", "select_blocks_adaptive",
           "cluster_attention_fwd_ragged", "ca_basic_workspace_bytes", "cluster_qk_basic", "ca_debug_attn_wait", "ca_debug_eigh",
           "ca_profile", "ca_profile_read", "rotary_axes", "ca_cache_workspace_bytes", "cache_append",
           "paged_attention_fwd", "ca_window_workspace_bytes", "window_attention_fwd")


class CaProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("n_q", ctypes.c_int32),
                ("n_k", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("cluster_q", ctypes.c_int32), ("cluster_k", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("compensate", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("flags", ctypes.c_int32)]

    @property
    def n_qc(self) -> int:
        return -(-self.n_q // self.cluster_q)

    @property
    def n_kc(self) -> int:
        return -(-self.n_k // self.cluster_k)

    def copy(self, **kw) -> "CaProblem":
        vals = {f: getattr(self, f) for f, _ in self._fields_}
        vals.update(kw)
        return CaProblem(**vals)


class CaRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64)]


class CaRotary(ctypes.Structure):
    _fields_ = [("axes", ctypes.c_int32), ("pairs", ctypes.c_int32 * 4), ("adjacent", ctypes.c_int32),
                ("freq", ctypes.POINTER(ctypes.c_double))]


class CaCache(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("page_rows", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("pages_per_sequence", ctypes.c_int32), ("left", ctypes.c_int32),
                ("sinks", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class CaWindow(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("n_q", ctypes.c_int32), ("n_k", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("left", ctypes.c_int32), ("right", ctypes.c_int32),
                ("sinks", ctypes.c_int32), ("softmax_scale", ctypes.c_float), ("flags", ctypes.c_int32)]


class ClusterAttnError(RuntimeError):
    pass


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libclusterattn.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ClusterAttnError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2608_26965_b200.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    pp = ctypes.POINTER(CaProblem)
    lib.ca_workspace_bytes.argtypes = [pp, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.ca_workspace_bytes.restype = ctypes.c_int
    lib.cluster_qk.argtypes = [pp] + [vp] * 16 + [sz, vp]
    lib.cluster_qk.restype = ctypes.c_int
    lib.select_blocks.argtypes = [pp, vp, vp, vp, vp, sz, vp]
    lib.select_blocks.restype = ctypes.c_int
    lib.cluster_attention_fwd.argtypes = [pp] + [vp] * 11 + [sz, vp]
    lib.cluster_attention_fwd.restype = ctypes.c_int
    lib.select_blocks_adaptive.argtypes = [pp, vp, vp, vp, ctypes.c_float, ctypes.c_int32, vp, vp, vp, sz, vp]
    lib.select_blocks_adaptive.restype = ctypes.c_int
    lib.cluster_attention_fwd_ragged.argtypes = [pp] + [vp] * 8 + [ctypes.c_int32] + [vp] * 4 + [sz, vp]
    lib.cluster_attention_fwd_ragged.restype = ctypes.c_int
    lib.ca_basic_workspace_bytes.argtypes = [pp, ctypes.POINTER(sz), ctypes.POINTER(ctypes.c_int32),
                                             ctypes.POINTER(ctypes.c_int32)]
    lib.ca_basic_workspace_bytes.restype = ctypes.c_int
    lib.cluster_qk_basic.argtypes = [pp] + [vp] * 5 + [ctypes.c_int32] + [vp] * 13 + [sz, vp]
    lib.cluster_qk_basic.restype = ctypes.c_int
    lib.ca_last_status.argtypes = [vp]
    lib.ca_last_status.restype = ctypes.c_int
    lib.ca_attn_recomputed.argtypes = [vp]
    lib.ca_attn_recomputed.restype = ctypes.c_int
    lib.ca_version.argtypes = []
    lib.ca_version.restype = ctypes.c_char_p
    lib.ca_kernel_launches.argtypes = []
    lib.ca_kernel_launches.restype = ctypes.c_ulonglong
    lib.cluster_attention_fwd_static.argtypes = [pp] + [vp] * 10 + [vp]
    lib.cluster_attention_fwd_static.restype = ctypes.c_int
    lib.ca_static_scratch_bytes.argtypes = []
    lib.ca_static_scratch_bytes.restype = ctypes.c_size_t
    lib.ca_static_last_status.argtypes = []
    lib.ca_static_last_status.restype = ctypes.c_int
    lib.ca_debug_attn_wait.argtypes = [ctypes.c_longlong, ctypes.c_int]
    lib.ca_debug_attn_wait.restype = None
    lib.ca_debug_eigh.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_void_p]
    lib.ca_debug_eigh.restype = ctypes.c_int
    lib.ca_profile.argtypes = [ctypes.c_int]
    lib.ca_profile.restype = ctypes.c_int
    lib.ca_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float),
                                    ctypes.POINTER(ctypes.c_int)]
    lib.ca_profile_read.restype = ctypes.c_int
    i32, i64, rp = ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(CaRows)
    lib.rotary_axes.argtypes = [ctypes.POINTER(CaRotary)] + [i32] * 7 + [rp, rp, vp, i64, rp, rp, vp]
    lib.rotary_axes.restype = ctypes.c_int
    lib.ca_cache_workspace_bytes.argtypes = [ctypes.POINTER(CaCache), ctypes.POINTER(sz)]
    lib.ca_cache_workspace_bytes.restype = ctypes.c_int
    lib.cache_append.argtypes = [ctypes.POINTER(CaCache), i32, rp, rp, vp, vp, vp, ctypes.POINTER(CaRotary), vp, i64, vp, vp, vp, sz, vp]
    lib.cache_append.restype = ctypes.c_int
    lib.paged_attention_fwd.argtypes = [ctypes.POINTER(CaCache), rp, vp, vp, vp, i32, vp, rp, vp, vp, sz, vp]
    lib.paged_attention_fwd.restype = ctypes.c_int
    lib.ca_window_workspace_bytes.argtypes = [ctypes.POINTER(CaWindow), ctypes.POINTER(sz)]
    lib.ca_window_workspace_bytes.restype = ctypes.c_int
    lib.window_attention_fwd.argtypes = [ctypes.POINTER(CaWindow), rp, rp, rp, vp, vp, rp, vp, vp, sz, vp]
    lib.window_attention_fwd.restype = ctypes.c_int
    _lib = lib
    return lib


def profile(enable: bool) -> None:
    """Switches the library's per-kernel-group timers on or off (ca_profile)."""
    _check(load_library().ca_profile(1 if enable else 0), "ca_profile")


def profile_read() -> Dict[str, Dict[str, float]]:
    """Device time in ms and number of timed scopes per kernel group since the timers were switched
    on or last read (ca_profile_read; synchronises the device)."""
    lib = load_library()
    n = 16
    names = (ctypes.c_char_p * n)()
    ms = (ctypes.c_float * n)()
    scopes = (ctypes.c_int * n)()
    got = lib.ca_profile_read(n, names, ms, scopes)
    if got < 0:
        _check(-got, "ca_profile_read")
    return {names[i].decode(): {"ms": float(ms[i]), "scopes": int(scopes[i])} for i in range(got)}


def kernel_launches() -> int:
    """Kernels the library has enqueued since it was loaded."""
    return int(load_library().ca_kernel_launches())


def _check(rc: int, what: str) -> None:
    if rc != CA_OK:
        raise ClusterAttnError(f"{what} failed: {ERRORS.get(rc, rc)}")


def _require_cuda(t: torch.Tensor, name: str) -> None:
    if not t.is_cuda:
        raise ClusterAttnError(f"{name} must be a CUDA tensor (no CPU path exists)")
    if not t.is_contiguous():
        raise ClusterAttnError(f"{name} must be contiguous")


_SAME = contextlib.nullcontext()


def _on(stream: Optional[torch.cuda.Stream]):
    """Where a call makes buffers: in order with what its stream does."""
    return _SAME if stream is None else torch.cuda.stream(stream)


def _filled(device: torch.device) -> None:
    """Waits for the fills of buffers that were just made: the calls take any stream, and nothing orders it behind the one that
    the buffers were made on.  (In a capture nothing runs yet, and the fills are part of it.)"""
    stream = torch.cuda.current_stream(device)
    with torch.cuda.device(device):
        capturing = torch.cuda.is_current_stream_capturing()
    if not capturing:
        stream.synchronize()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream_ptr(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def torch_dtype(problem: CaProblem) -> torch.dtype:
    return torch.bfloat16 if problem.dtype == CA_DTYPE_BF16 else torch.float32


def _numbers32(**numbers) -> None:
    """ctypes takes the lower 32 bits of what does not fit an int32 without a word: a left bound of 2^32 would be one of 0."""
    for name, x in numbers.items():
        if not -2 ** 31 <= x < 2 ** 31:
            raise ClusterAttnError(f"{name} must be a 32-bit number, not {x}")


def make_problem(batch: int, heads: int, n_q: int, n_k: int, head_dim: int, dtype: str, cluster_q: int,
                 cluster_k: int, keep: int, compensate: bool = True, softmax_scale: float = 0.0,
                 flags: int = 0) -> CaProblem:
    code = {"fp32": CA_DTYPE_FP32, "bf16": CA_DTYPE_BF16}[dtype]
    _numbers32(batch=batch, heads=heads, n_q=n_q, n_k=n_k, head_dim=head_dim, cluster_q=cluster_q, cluster_k=cluster_k, keep=keep,
               flags=flags)
    return CaProblem(batch, heads, n_q, n_k, head_dim, code, cluster_q, cluster_k, keep,
                     1 if compensate else 0, float(softmax_scale), flags)


def problem_from_workload(w, heads: Optional[int] = None, **kw) -> CaProblem:
    args = dict(batch=1, heads=heads if heads is not None else w.heads, n_q=w.n_q, n_k=w.n_k,
                head_dim=w.head_dim, dtype=w.dtype, cluster_q=w.cluster, cluster_k=w.cluster, keep=w.keep,
                compensate=w.compensate)
    args.update(kw)
    return make_problem(**args)


def debug_eigh(A: torch.Tensor, stream=None):
    """ca_debug_eigh of the C library: A [count, d, d] float64 symmetric (CUDA).  Returns
    (W [count, d, d] float32 with eigenvector t in column t, evals [count, d] float64, descending)."""
    _require_cuda(A, "A")
    if A.dtype != torch.float64 or A.dim() != 3 or A.shape[1] != A.shape[2]:
        raise ClusterAttnError("A must be [count, d, d] float64")
    lib = load_library()
    count, d = int(A.shape[0]), int(A.shape[1])
    W = torch.empty((count, d, d), dtype=torch.float32, device=A.device)
    ev = torch.empty((count, d), dtype=torch.float64, device=A.device)
    _check(lib.ca_debug_eigh(_ptr(A), count, d, _ptr(W), _ptr(ev), _stream_ptr(stream)), "ca_debug_eigh")
    return W, ev


def workspace_bytes(problem: CaProblem) -> Dict[str, int]:
    lib = load_library()
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.ca_workspace_bytes(ctypes.byref(problem), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
           "ca_workspace_bytes")
    return {"cluster": a.value, "select": b.value, "attn": c.value}


class Plan:
    """Device buffers for one problem shape: outputs of each stage and the
    workspaces the library asks for.  Holds memory only; all compute is in the
    library calls."""

    def __init__(self, problem: CaProblem, device: str = "cuda:0", keep_y: bool = False):
        if not torch.cuda.is_available():
            raise ClusterAttnError("no CUDA device: libclusterattn has no CPU path")
        load_library()
        self.problem = problem = problem.copy()             # (the caller's may change; the buffers here do not)
        self.device = torch.device(device)
        p = problem
        dt = torch_dtype(p)
        B, H, D = p.batch, p.heads, p.head_dim
        dev = self.device
        i32, f32 = torch.int32, torch.float32
        self.perm_q = torch.empty((B, H, p.n_q), dtype=i32, device=dev)
        self.perm_k = torch.empty((B, H, p.n_k), dtype=i32, device=dev)
        self.Qp = torch.empty((B, H, p.n_qc * p.cluster_q, D), dtype=dt, device=dev)
        self.Kp = torch.empty((B, H, p.n_kc * p.cluster_k, D), dtype=dt, device=dev)
        self.Vp = torch.empty((B, H, p.n_kc * p.cluster_k, D), dtype=dt, device=dev)
        self.cq = torch.empty((B, H, p.n_qc, D), dtype=f32, device=dev)
        self.ck = torch.empty((B, H, p.n_kc, D), dtype=f32, device=dev)
        self.cv = torch.empty((B, H, p.n_kc, D), dtype=f32, device=dev)
        self.count_q = torch.empty((B, H, p.n_qc), dtype=i32, device=dev)
        self.count_k = torch.empty((B, H, p.n_kc), dtype=i32, device=dev)
        self.block_idx = torch.empty((B, H, p.n_qc, p.keep), dtype=i32, device=dev)
        self.block_idx_ragged = None
        self.keep_count = None
        self.O = torch.empty((B, H, p.n_q, D), dtype=dt, device=dev)
        self.lse = torch.empty((B, H, p.n_q), dtype=f32, device=dev)
        self.Yq = torch.empty((B, H, p.n_q, D), dtype=f32, device=dev) if keep_y else None
        self.Yk = torch.empty((B, H, p.n_k, D), dtype=f32, device=dev) if keep_y else None
        sizes = workspace_bytes(p)
        self.ws = {k: torch.zeros(max(v, 256), dtype=torch.uint8, device=dev) for k, v in sizes.items()}
        _filled(dev)

    # -- the three entry points ------------------------------------------------
    def cluster_qk(self, Q, K, V, Yq=None, Yk=None, stream=None):
        """cluster_qk of the C library.  With Yq/Yk given and CA_Y_IN set in the
        problem's flags the split coordinates are taken from the caller."""
        p = self.problem
        for name, t in (("Q", Q), ("K", K), ("V", V)):
            _require_cuda(t, name)
        yq = Yq if Yq is not None else self.Yq
        yk = Yk if Yk is not None else self.Yk
        if p.flags & CA_Y_IN:
            _require_cuda(yq, "Yq")
            _require_cuda(yk, "Yk")
        lib = load_library()
        ws = self.ws["cluster"]
        rc = lib.cluster_qk(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(self.perm_q), _ptr(self.perm_k),
                            _ptr(self.Qp), _ptr(self.Kp), _ptr(self.Vp), _ptr(self.cq), _ptr(self.ck),
                            _ptr(self.cv), _ptr(self.count_q), _ptr(self.count_k), _ptr(yq), _ptr(yk),
                            _ptr(ws), ws.numel(), _stream_ptr(stream))
        _check(rc, "cluster_qk")
        return self

    def select_blocks(self, cq=None, ck=None, stream=None):
        lib = load_library()
        cq = self.cq if cq is None else cq
        ck = self.ck if ck is None else ck
        _require_cuda(cq, "cq")
        _require_cuda(ck, "ck")
        ws = self.ws["select"]
        rc = lib.select_blocks(ctypes.byref(self.problem), _ptr(cq), _ptr(ck), _ptr(self.block_idx), _ptr(ws),
                               ws.numel(), _stream_ptr(stream))
        _check(rc, "select_blocks")
        return self.block_idx

    def cluster_attention_fwd(self, Qp=None, Kp=None, Vp=None, ck=None, cv=None, count_k=None,
                              block_idx=None, perm_q=None, want_lse=True, stream=None):
        lib = load_library()
        args = [self.Qp if Qp is None else Qp, self.Kp if Kp is None else Kp, self.Vp if Vp is None else Vp,
                self.ck if ck is None else ck, self.cv if cv is None else cv,
                self.count_k if count_k is None else count_k,
                self.block_idx if block_idx is None else block_idx,
                self.perm_q if perm_q is None else perm_q]
        for i, t in enumerate(args):
            _require_cuda(t, f"arg{i}")
        ws = self.ws["attn"]
        rc = lib.cluster_attention_fwd(ctypes.byref(self.problem), *[_ptr(t) for t in args], _ptr(self.O),
                                       _ptr(self.lse if want_lse else None), _ptr(ws), ws.numel(),
                                       _stream_ptr(stream))
        _check(rc, "cluster_attention_fwd")
        return self.O, (self.lse if want_lse else None)

    def basic_noise_rows(self):
        """Rows of normal deviates per head that cluster_qk_basic reads (queries, keys)."""
        lib = load_library()
        b, rq, rk = ctypes.c_size_t(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib.ca_basic_workspace_bytes(ctypes.byref(self.problem), ctypes.byref(b), ctypes.byref(rq),
                                            ctypes.byref(rk)), "ca_basic_workspace_bytes")
        return rq.value, rk.value, b.value

    def cluster_qk_basic(self, Q, K, V, noise_q, noise_k, iterations: int = 3, A_q=None, A_k=None, stream=None):
        """cluster_qk_basic of the C library: basic recursive splitting with the metric injected into
        the power iteration.  noise_q/noise_k: normal deviates [B,H,rows,d] (rows from basic_noise_rows).
        A_q/A_k are inputs when the problem has CA_METRIC_IN, otherwise they are written."""
        lib = load_library()
        p = self.problem
        for name, t in (("Q", Q), ("K", K), ("V", V), ("noise_q", noise_q), ("noise_k", noise_k)):
            _require_cuda(t, name)
        rq, rk, nbytes = self.basic_noise_rows()
        if tuple(noise_q.shape[-2:]) != (rq, p.head_dim) or tuple(noise_k.shape[-2:]) != (rk, p.head_dim):
            raise ClusterAttnError(f"noise must be [B,H,{rq},{p.head_dim}] and [B,H,{rk},{p.head_dim}]")
        if p.flags & CA_METRIC_IN and (A_q is None or A_k is None):
            raise ClusterAttnError("CA_METRIC_IN needs A_q and A_k")
        shape = (p.batch, p.heads, p.head_dim, p.head_dim)
        with _on(stream):
            self.A_q = A_q if A_q is not None else torch.empty(shape, dtype=torch.float32, device=self.device)
            self.A_k = A_k if A_k is not None else torch.empty(shape, dtype=torch.float32, device=self.device)
            if self.ws.get("basic") is None or self.ws["basic"].numel() < nbytes:
                self.ws["basic"] = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        ws = self.ws["basic"]
        rc = lib.cluster_qk_basic(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(noise_q), _ptr(noise_k),
                                  int(iterations), _ptr(self.A_q), _ptr(self.A_k), _ptr(self.perm_q),
                                  _ptr(self.perm_k), _ptr(self.Qp), _ptr(self.Kp), _ptr(self.Vp), _ptr(self.cq),
                                  _ptr(self.ck), _ptr(self.cv), _ptr(self.count_q), _ptr(self.count_k), _ptr(ws),
                                  ws.numel(), _stream_ptr(stream))
        _check(rc, "cluster_qk_basic")
        return self

    def select_blocks_adaptive(self, recall: float, min_count: int = 16, cq=None, ck=None, count_k=None,
                               stream=None):
        """Adaptive assignment: returns (block_idx [B,H,n_qc,n_kc] padded with -1, keep_count [B,H,n_qc])."""
        lib = load_library()
        cq = self.cq if cq is None else cq
        ck = self.ck if ck is None else ck
        count_k = self.count_k if count_k is None else count_k
        for name, t in (("cq", cq), ("ck", ck), ("count_k", count_k)):
            _require_cuda(t, name)
        pr = self.problem
        if getattr(self, "block_idx_ragged", None) is None:
            with _on(stream):
                self.block_idx_ragged = torch.empty((pr.batch, pr.heads, pr.n_qc, pr.n_kc), dtype=torch.int32,
                                                    device=self.device)
                self.keep_count = torch.empty((pr.batch, pr.heads, pr.n_qc), dtype=torch.int32, device=self.device)
        ws = self.ws["select"]
        rc = lib.select_blocks_adaptive(ctypes.byref(pr), _ptr(cq), _ptr(ck), _ptr(count_k), float(recall),
                                        int(min_count), _ptr(self.block_idx_ragged), _ptr(self.keep_count),
                                        _ptr(ws), ws.numel(), _stream_ptr(stream))
        _check(rc, "select_blocks_adaptive")
        return self.block_idx_ragged, self.keep_count

    def cluster_attention_fwd_ragged(self, block_idx=None, keep_count=None, Qp=None, Kp=None, Vp=None, ck=None,
                                     cv=None, count_k=None, perm_q=None, want_lse=True, stream=None):
        lib = load_library()
        block_idx = self.block_idx_ragged if block_idx is None else block_idx
        keep_count = self.keep_count if keep_count is None else keep_count
        args = [self.Qp if Qp is None else Qp, self.Kp if Kp is None else Kp, self.Vp if Vp is None else Vp,
                self.ck if ck is None else ck, self.cv if cv is None else cv,
                self.count_k if count_k is None else count_k, block_idx, keep_count]
        perm_q = self.perm_q if perm_q is None else perm_q
        for i, t in enumerate(args + [perm_q]):
            _require_cuda(t, f"arg{i}")
        ws = self.ws["attn"]
        rc = lib.cluster_attention_fwd_ragged(ctypes.byref(self.problem), *[_ptr(t) for t in args],
                                              int(block_idx.shape[-1]), _ptr(perm_q), _ptr(self.O),
                                              _ptr(self.lse if want_lse else None), _ptr(ws), ws.numel(),
                                              _stream_ptr(stream))
        _check(rc, "cluster_attention_fwd_ragged")
        return self.O, (self.lse if want_lse else None)

    def _turned(self, Q, K, rotary, positions_q, positions_k, stream):
        """Q and K turned by their positions (rotary_axes), in buffers of the plan."""
        p, dt = self.problem, torch_dtype(self.problem)
        if getattr(self, "Qr", None) is None:
            with _on(stream):
                self.Qr = torch.empty((p.batch, p.heads, p.n_q, p.head_dim), dtype=dt, device=self.device)
                self.Kr = torch.empty((p.batch, p.heads, p.n_k, p.head_dim), dtype=dt, device=self.device)
        if positions_k is None and p.n_q == p.n_k:
            return rotary_axes(rotary, Q, K, positions_q, out_q=self.Qr, out_k=self.Kr, stream=stream)
        rotary_axes(rotary, Q, None, positions_q, out_q=self.Qr, stream=stream)
        rotary_axes(rotary, K, None, positions_k, out_q=self.Kr, stream=stream)
        return self.Qr, self.Kr

    @staticmethod
    def _no_positions(positions_q, positions_k):
        if positions_q is not None or positions_k is not None:
            raise ClusterAttnError("positions without rotary")

    def forward_adaptive(self, Q, K, V, recall: float, min_count: int = 16, want_lse=False, stream=None, rotary=None,
                         positions_q=None, positions_k=None):
        if rotary is not None:
            Q, K = self._turned(Q, K, rotary, positions_q, positions_k, stream)
        else:
            self._no_positions(positions_q, positions_k)
        self.cluster_qk(Q, K, V, stream=stream)
        self.select_blocks_adaptive(recall, min_count, stream=stream)
        return self.cluster_attention_fwd_ragged(want_lse=want_lse, stream=stream)

    def forward(self, Q, K, V, want_lse=False, stream=None, rotary=None, positions_q=None, positions_k=None):
        """The whole hot path: clustering, block selection, attention.  With `rotary` (a Rotary) the queries and
        keys are turned first, by positions_q and positions_k [batch or 1, n, axes] int32 (positions_k None: the
        queries' own); Q and K may then be strided."""
        if rotary is not None:
            Q, K = self._turned(Q, K, rotary, positions_q, positions_k, stream)
        else:
            self._no_positions(positions_q, positions_k)
        self.cluster_qk(Q, K, V, stream=stream)
        self.select_blocks(stream=stream)
        return self.cluster_attention_fwd(want_lse=want_lse, stream=stream)[0]

    def last_status(self) -> Dict[str, int]:
        lib = load_library()
        return {k: lib.ca_last_status(_ptr(v)) for k, v in self.ws.items()}

    def recomputed_clusters(self) -> int:
        """Query clusters that the second pass of the attention calls on this plan has recomputed
        with the fp32 kernel, summed over all calls since the plan was made (ca_attn_recomputed)."""
        lib = load_library()
        n = lib.ca_attn_recomputed(_ptr(self.ws["attn"]))
        if n < 0:
            _check(-n, "ca_attn_recomputed")
        return n


# -- streams of tokens: rotary positions, a cache in pages, sliding windows -----------
# These calls take [batch, heads, rows, head_dim] tensors by strides (the last dimension dense, strides of
# 16 bytes), run on the device of their tensors whatever the current one is, and by default on its current stream.
_CODES = {"fp32": CA_DTYPE_FP32, "bf16": CA_DTYPE_BF16}
_TORCH = {CA_DTYPE_FP32: torch.float32, CA_DTYPE_BF16: torch.bfloat16}
_OF_TORCH = {torch.float32: CA_DTYPE_FP32, torch.bfloat16: CA_DTYPE_BF16}


def _code(dtype: str) -> int:
    if dtype not in _CODES:
        raise ClusterAttnError(f"dtype must be one of {sorted(_CODES)}, not {dtype!r}")
    return _CODES[dtype]


def _rows(t: torch.Tensor, name: str, shape, dtype: torch.dtype, device: torch.device) -> CaRows:
    """A [batch, heads, rows, head_dim] tensor of that shape, type and device as the library takes it."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ClusterAttnError(f"{name} must be a CUDA tensor (no CPU path exists)")
    if t.dtype != dtype or t.shape != shape or t.device != device:
        raise ClusterAttnError(f"{name} must be {dtype} {list(shape)} on {device}, not {t.dtype} {list(t.shape)} on {t.device}")
    sb, sh, sn, sd = t.stride()
    if sd != 1:
        raise ClusterAttnError(f"{name}: the last dimension must be dense")
    return CaRows(t.data_ptr(), sb, sh, sn)


def _int32(t: Optional[torch.Tensor], name: str, shape, device: torch.device):
    """Address of a dense int32 tensor of that shape, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise ClusterAttnError(f"{name} must be a tensor on {device}")
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ClusterAttnError(f"{name} must be a contiguous int32 tensor {list(shape)}, not {t.dtype} {list(t.shape)}")
    return t.data_ptr()


def _cuda_device(device) -> torch.device:
    d = torch.device(device)
    if d.type != "cuda" or not torch.cuda.is_available():
        raise ClusterAttnError("no CUDA device: libclusterattn has no CPU path")
    return d if d.index is not None else torch.device("cuda", torch.cuda.current_device())


# address of the current stream of a device; torch's own shortcut takes 0.1 us, the stream object 2.2
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _call(fn, what: str, device: torch.device, stream: Optional[torch.cuda.Stream], *args) -> None:
    """A library call on `stream` (default: the device's current one) with the device current."""
    if stream is None:
        handle = _raw_stream(device.index)
    else:
        if stream.device != device:
            raise ClusterAttnError(f"{what}: the stream is on {stream.device}, the tensors on {device}")
        handle = stream.cuda_stream
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, handle)
    if rc != CA_OK:
        _check(rc, what)


class Rotary:
    """Rotary positions: pairs[a] pairs of channels turn with axis a of a position, by `frequencies` (radians
    per step, one for every pair), or theta ** (-i / pairs[a]) for pair i of an axis.  adjacent: pair c is
    channels (2c, 2c + 1), otherwise (c, R + c) with R the number of pairs."""

    def __init__(self, head_dim: int, pairs, theta: float = 10000.0, frequencies=None, adjacent: bool = True):
        pairs = [int(p) for p in pairs]
        if not 1 <= len(pairs) <= 4 or min(pairs) < 0 or not 1 <= sum(pairs) <= head_dim // 2:
            raise ClusterAttnError(f"pairs must be 1 to 4 counts, 1 to {head_dim // 2} in all, not {pairs}")
        if frequencies is None:
            frequencies = [theta ** (-i / n) for n in pairs for i in range(n)]
        frequencies = [float(f) for f in frequencies]
        if len(frequencies) != sum(pairs) or not all(abs(f) <= 2.0 ** 32 for f in frequencies):
            raise ClusterAttnError(f"frequencies must be {sum(pairs)} numbers of at most 2^32")
        self.head_dim, self.pairs, self.frequencies, self.adjacent = int(head_dim), pairs, frequencies, bool(adjacent)
        self._freq = (ctypes.c_double * len(frequencies))(*frequencies)
        self._struct = CaRotary(len(pairs), (ctypes.c_int32 * 4)(*pairs), 1 if adjacent else 0,
                                ctypes.cast(self._freq, ctypes.POINTER(ctypes.c_double)))

    def _positions(self, positions, batch: int, n: int, device: torch.device):
        """Pointer and batch stride of positions [batch, n, axes], or [1, n, axes] for the whole batch."""
        if not isinstance(positions, torch.Tensor) or positions.dim() != 3:
            raise ClusterAttnError("positions must be a [batch or 1, n, axes] tensor")
        axes = len(self.pairs)
        shape = (1 if positions.shape[0] == 1 else batch, n, axes)
        return _int32(positions, "positions", shape, device), (0 if shape[0] == 1 else n * axes)


def rotary_axes(rotary: Rotary, q, k, positions, inverse: bool = False, out_q=None, out_k=None, stream=None):
    """rotary_axes of the C library: q [batch, heads, n, head_dim] and k (or None) turned by their positions
    [batch or 1, n, axes] int32.  Returns (q', k'): new dense tensors, or out_q / out_k, which may be q and k."""
    if not isinstance(q, torch.Tensor) or q.dim() != 4 or q.dtype not in _OF_TORCH:
        raise ClusterAttnError("q must be a [batch, heads, n, head_dim] tensor of float32 or bfloat16")
    if not q.is_cuda:
        raise ClusterAttnError("q must be a CUDA tensor (no CPU path exists)")
    device, dtype, shape = q.device, q.dtype, q.shape
    B, H, n, D = shape
    if D != rotary.head_dim:
        raise ClusterAttnError(f"q has head_dim {D}, the rotary positions {rotary.head_dim}")
    pos, pos_b = rotary._positions(positions, B, n, device)
    a, b, d, Hk = _rows(q, "q", shape, dtype, device), None, None, 0
    if k is not None:
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ClusterAttnError("k must be a [batch, heads, n, head_dim] tensor")
        Hk = k.shape[1]
        shape_k = (B, Hk, n, D)
        b = _rows(k, "k", shape_k, dtype, device)
    elif out_k is not None:
        raise ClusterAttnError("out_k without k")
    c = _rows(out_q, "out_q", shape, dtype, device) if out_q is not None else None
    if k is not None and out_k is not None:
        d = _rows(out_k, "out_k", shape_k, dtype, device)
    if c is None or (k is not None and d is None):
        # new dense memory
        with _on(stream):
            if c is None:
                out_q = q.new_empty(shape)
                c = CaRows(out_q.data_ptr(), H * n * D, n * D, D)
            if k is not None and d is None:
                out_k = q.new_empty(shape_k)
                d = CaRows(out_k.data_ptr(), Hk * n * D, n * D, D)
    _call(load_library().rotary_axes, "rotary_axes", device, stream, rotary._struct, B, H, Hk, n, D, _OF_TORCH[dtype],
          1 if inverse else 0, a, b, pos, pos_b, c, d)
    return out_q, out_k


def make_cache_problem(batch: int, heads_q: int, heads_kv: int, head_dim: int, dtype: str, page_rows: int, pages: int,
                       pages_per_sequence: int, left: int = -1, sinks: int = 0, softmax_scale: float = 0.0) -> CaCache:
    _numbers32(batch=batch, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim, page_rows=page_rows, pages=pages,
               pages_per_sequence=pages_per_sequence, left=left, sinks=sinks)
    return CaCache(batch, heads_q, heads_kv, head_dim, _code(dtype), page_rows, pages, pages_per_sequence, left, sinks,
                   float(softmax_scale))


class PagedCache:
    """Keys and values of `batch` sequences in pages: pools K_pages, V_pages [pages, heads_kv, page_rows, head_dim],
    page_table [batch, pages_per_sequence] and lengths [batch] int32 (made here, zeros, where they are not given), and the
    workspace and outputs of the calls.  The program that owns the cache writes page_table and lengths; the
    calls only read them."""

    def __init__(self, problem: CaCache, device: str = "cuda:0", K_pages=None, V_pages=None, page_table=None, lengths=None):
        self.device = dev = _cuda_device(device)
        self.problem = p = CaCache.from_buffer_copy(problem)             # (as in Plan)
        lib = load_library()
        size = ctypes.c_size_t()
        _check(lib.ca_cache_workspace_bytes(ctypes.byref(p), ctypes.byref(size)), "ca_cache_workspace_bytes")
        self.dtype = _TORCH[p.dtype]
        pool = (p.pages, p.heads_kv, p.page_rows, p.head_dim)
        self._K_pages = torch.zeros(pool, dtype=self.dtype, device=dev) if K_pages is None else K_pages
        self._V_pages = torch.zeros(pool, dtype=self.dtype, device=dev) if V_pages is None else V_pages
        self._page_table = (torch.zeros((p.batch, p.pages_per_sequence), dtype=torch.int32, device=dev)
                            if page_table is None else page_table)
        self._lengths = torch.zeros((p.batch,), dtype=torch.int32, device=dev) if lengths is None else lengths
        for name, t in (("K_pages", self._K_pages), ("V_pages", self._V_pages)):
            _rows(t, name, pool, self.dtype, dev)
            if not t.is_contiguous():
                raise ClusterAttnError(f"{name} must be contiguous")
        for name, t, shape in (("lengths", self._lengths, (p.batch,)), ("page_table", self._page_table, (p.batch, p.pages_per_sequence))):
            if _int32(t, name, shape, dev) is None:
                raise ClusterAttnError(f"{name} is missing")
        self.O = torch.zeros((p.batch, p.heads_q, 1, p.head_dim), dtype=self.dtype, device=dev)
        self.lse = torch.zeros((p.batch, p.heads_q, 1), dtype=torch.float32, device=dev)
        self.ws = torch.zeros(size.value, dtype=torch.uint8, device=dev)
        _filled(dev)

    # the tensors of the cache: written into by the program, and the same ones for the life of the cache
    K_pages = property(lambda self: self._K_pages)
    V_pages = property(lambda self: self._V_pages)
    page_table = property(lambda self: self._page_table)
    lengths = property(lambda self: self._lengths)

    def cache_append(self, K, V, count=None, rotary: Optional[Rotary] = None, positions=None, stream=None):
        """cache_append of the C library: rows of K and V [batch, heads_kv, n, head_dim] (of sequence b the first
        count[b]) behind the lengths[b] rows that are there, K turned by `rotary` at `positions` on the way."""
        p = self.problem
        if not isinstance(K, torch.Tensor) or K.dim() != 4:
            raise ClusterAttnError("K must be a [batch, heads_kv, n, head_dim] tensor")
        n = K.shape[2]
        shape = (p.batch, p.heads_kv, n, p.head_dim)
        k, v = _rows(K, "K", shape, self.dtype, self.device), _rows(V, "V", shape, self.dtype, self.device)
        pos, pos_b, rot = None, 0, None
        if rotary is not None:
            if rotary.head_dim != p.head_dim:
                raise ClusterAttnError(f"the cache has head_dim {p.head_dim}, the rotary positions {rotary.head_dim}")
            pos, pos_b = rotary._positions(positions, p.batch, n, self.device)
            rot = rotary._struct
        elif positions is not None:
            raise ClusterAttnError("positions without rotary")
        _call(load_library().cache_append, "cache_append", self.device, stream, p, n, k, v, self._lengths.data_ptr(),
              _int32(count, "count", (p.batch,), self.device), self._page_table.data_ptr(), rot, pos, pos_b, self._K_pages.data_ptr(),
              self._V_pages.data_ptr(), self.ws.data_ptr(), self.ws.numel())

    def paged_attention_fwd(self, Q, appended: int = 0, out=None, want_lse: bool = True, stream=None):
        """paged_attention_fwd of the C library: Q [batch, heads_q, 1, head_dim] against lengths[b] + appended
        rows.  Returns (O, lse [batch, heads_q, 1] or None): the cache's buffers, O or `out`."""
        p = self.problem
        shape = (p.batch, p.heads_q, 1, p.head_dim)
        _numbers32(appended=appended)
        out = self.O if out is None else out
        q, o = _rows(Q, "Q", shape, self.dtype, self.device), _rows(out, "out", shape, self.dtype, self.device)
        lse = self.lse if want_lse else None
        _call(load_library().paged_attention_fwd, "paged_attention_fwd", self.device, stream, p, q, self._K_pages.data_ptr(),
              self._V_pages.data_ptr(), self._lengths.data_ptr(), int(appended), self._page_table.data_ptr(), o, None if lse is None else lse.data_ptr(), self.ws.data_ptr(), self.ws.numel())
        return out, lse

    def last_status(self) -> int:
        """Status word that the last call left (ca_last_status; synchronises the device)."""
        with torch.cuda.device(self.device):
            return load_library().ca_last_status(_ptr(self.ws))


def make_window_problem(batch: int, heads_q: int, heads_kv: int, n_q: int, n_k: int, head_dim: int, dtype: str, left: int,
                        right: int, sinks: int = 0, softmax_scale: float = 0.0, flags: int = 0) -> CaWindow:
    _numbers32(batch=batch, heads_q=heads_q, heads_kv=heads_kv, n_q=n_q, n_k=n_k, head_dim=head_dim, left=left, right=right, sinks=sinks,
               flags=flags)
    return CaWindow(batch, heads_q, heads_kv, n_q, n_k, head_dim, _code(dtype), left, right, sinks, float(softmax_scale), flags)


class WindowPlan:
    """Outputs and workspace of attention over a sliding window for one problem shape."""

    def __init__(self, problem: CaWindow, device: str = "cuda:0"):
        self.device = dev = _cuda_device(device)
        self.problem = p = CaWindow.from_buffer_copy(problem)
        size = ctypes.c_size_t()
        _check(load_library().ca_window_workspace_bytes(ctypes.byref(p), ctypes.byref(size)), "ca_window_workspace_bytes")
        self.dtype = _TORCH[p.dtype]
        self.O = torch.zeros((p.batch, p.heads_q, p.n_q, p.head_dim), dtype=self.dtype, device=dev)
        self.lse = torch.zeros((p.batch, p.heads_q, p.n_q), dtype=torch.float32, device=dev)
        self.ws = torch.zeros(size.value, dtype=torch.uint8, device=dev)
        _filled(dev)

    def window_attention_fwd(self, Q, K, V, len_q=None, len_k=None, out=None, want_lse: bool = True, stream=None):
        """window_attention_fwd of the C library.  Returns (O, lse or None): the plan's buffers, O or `out`; rows
        from len_q[b] on are left as they were."""
        p, dt, dev = self.problem, self.dtype, self.device
        out = self.O if out is None else out
        q = _rows(Q, "Q", (p.batch, p.heads_q, p.n_q, p.head_dim), dt, dev)
        k = _rows(K, "K", (p.batch, p.heads_kv, p.n_k, p.head_dim), dt, dev)
        v = _rows(V, "V", (p.batch, p.heads_kv, p.n_k, p.head_dim), dt, dev)
        o = _rows(out, "out", (p.batch, p.heads_q, p.n_q, p.head_dim), dt, dev)
        lse = self.lse if want_lse else None
        _call(load_library().window_attention_fwd, "window_attention_fwd", dev, stream, p, q, k, v,
              _int32(len_q, "len_q", (p.batch,), dev), _int32(len_k, "len_k", (p.batch,), dev), o,
              None if lse is None else lse.data_ptr(), self.ws.data_ptr(), self.ws.numel())
        return out, lse

    def last_status(self) -> int:
        """Status word that the last call left (ca_last_status; synchronises the device)."""
        with torch.cuda.device(self.device):
            return load_library().ca_last_status(_ptr(self.ws))


# -- functional forms with the C names ------------------------------------------
def cluster_qk(problem: CaProblem, Q, K, V, Yq=None, Yk=None, plan: Optional[Plan] = None) -> Plan:
    plan = plan or Plan(problem, device=str(Q.device), keep_y=Yq is None)
    return plan.cluster_qk(Q, K, V, Yq=Yq, Yk=Yk)


def select_blocks(problem: CaProblem, cq, ck, plan: Optional[Plan] = None):
    plan = plan or Plan(problem, device=str(cq.device))
    return plan.select_blocks(cq, ck)


def cluster_attention_fwd(problem: CaProblem, Qp, Kp, Vp, ck, cv, count_k, block_idx, perm_q,
                          plan: Optional[Plan] = None):
    plan = plan or Plan(problem, device=str(Qp.device))
    if tuple(block_idx.shape[-2:]) != (problem.n_qc, problem.keep):
        raise ClusterAttnError("block_idx must be [B,H,n_qc,keep]")
    return plan.cluster_attention_fwd(Qp, Kp, Vp, ck, cv, count_k, block_idx, perm_q)


def select_blocks_adaptive(problem: CaProblem, cq, ck, count_k, recall: float, min_count: int = 16,
                           plan: Optional[Plan] = None):
    plan = plan or Plan(problem, device=str(cq.device))
    return plan.select_blocks_adaptive(recall, min_count, cq, ck, count_k)


def cluster_attention_fwd_ragged(problem: CaProblem, Qp, Kp, Vp, ck, cv, count_k, block_idx, keep_count, perm_q,
                                 plan: Optional[Plan] = None):
    plan = plan or Plan(problem, device=str(Qp.device))
    return plan.cluster_attention_fwd_ragged(block_idx, keep_count, Qp, Kp, Vp, ck, cv, count_k, perm_q)


def cluster_attention_fwd_static(problem: CaProblem, Qp, Kp, Vp, ck, cv, count_k, block_idx, perm_q, O,
                                 lse=None, stream=None):
    """The attention stage for callers that cannot allocate device memory (no
    workspace argument: the library's fixed 32 MiB scratch array is used).  The
    caller passes every input and the output tensors; nothing is allocated here
    either.  Calls on one device share the scratch and must not overlap."""
    lib = load_library()
    args = [Qp, Kp, Vp, ck, cv, count_k, block_idx, perm_q, O]
    for i, t in enumerate(args):
        _require_cuda(t, f"arg{i}")
    rc = lib.cluster_attention_fwd_static(ctypes.byref(problem), *[_ptr(t) for t in args], _ptr(lse),
                                          _stream_ptr(stream))
    _check(rc, "cluster_attention_fwd_static")
    return O, lse


def static_scratch_bytes() -> int:
    return int(load_library().ca_static_scratch_bytes())


def default_scale(problem: CaProblem) -> float:
    return problem.softmax_scale if problem.softmax_scale > 0 else 1.0 / math.sqrt(problem.head_dim)
