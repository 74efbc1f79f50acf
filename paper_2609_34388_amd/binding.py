"""ctypes binding of librecguide.so (include/recguide.h).

Argument marshalling only: every computation runs in the library's HIP
kernels.  If the library is missing or cannot be loaded the first call
raises; there is no fallback.

Tensors are torch tensors on the GPU (bf16 as torch.bfloat16, indices as
torch.int32); per-request sizes for attention planning are host arrays
(numpy or CPU tensors).  Calls enqueue on the current torch stream unless a
``stream`` (torch.cuda.Stream or raw handle) is given and return without
synchronising.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from typing import Dict, Optional, Tuple

import numpy as np
import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librecguide.so")

RG_OK = 0
NOALLOC_SCRATCH_BYTES = 4 << 20  # RG_NOALLOC_SCRATCH_BYTES
_STATUS = {0: "ok", 1: "RG_ERR_NULL", 2: "RG_ERR_SHAPE", 3: "RG_ERR_UNSUPPORTED",
           4: "RG_ERR_WORKSPACE", 5: "RG_ERR_HIP", 6: "RG_ERR_WAIT"}


class RGError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_STATUS.get(status, status)} ({_lib().rg_status_string(status).decode()})")


class AttnLayout(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("sm_scale", ctypes.c_float),
                ("q_indptr", ctypes.c_void_p), ("n_verify", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p), ("page_indptr", ctypes.c_void_p),
                ("page_indices", ctypes.c_void_p)]


class BranchLayout(ctypes.Structure):
    _fields_ = [("branch_indptr", ctypes.c_void_p), ("prefix", ctypes.c_void_p),
                ("lead", ctypes.c_void_p), ("rows", ctypes.c_void_p)]


class BlockPolicy(ctypes.Structure):
    _fields_ = [("num_candidates", ctypes.c_int32), ("candidates", ctypes.c_void_p),
                ("num_s_bins", ctypes.c_int32), ("s_edges", ctypes.c_void_p), ("cost", ctypes.c_void_p),
                ("rho", ctypes.c_float), ("value", ctypes.c_void_p)]


class Rotation(ctypes.Structure):
    _fields_ = [("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p),
                ("positions", ctypes.c_void_p)]


class Window(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("sink", ctypes.c_int32)]


class EvictLayout(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("sink", ctypes.c_int32),
                ("recent", ctypes.c_int32), ("ctx_len", ctypes.c_void_p), ("keep", ctypes.c_void_p),
                ("tracked", ctypes.c_void_p), ("evicted", ctypes.c_void_p), ("page_indptr", ctypes.c_void_p),
                ("page_indices", ctypes.c_void_p)]


class AttnPlanInfo(ctypes.Structure):
    _fields_ = [("num_launches", ctypes.c_int32), ("chunk_keys", ctypes.c_int32),
                ("work_items", ctypes.c_int64), ("split_requests", ctypes.c_int64),
                ("partial_columns", ctypes.c_int64), ("workspace_bytes", ctypes.c_int64),
                ("persistent_launches", ctypes.c_int32), ("sync_words", ctypes.c_int32),
                ("sync_offset", ctypes.c_int64)]


class AttnLaunchInfo(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int32), ("joined_launches", ctypes.c_int32),
                ("merge_launches", ctypes.c_int32), ("run_keys", ctypes.c_int32), ("narrow", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("work_items", ctypes.c_int64), ("split_requests", ctypes.c_int64),
                ("partial_columns", ctypes.c_int64), ("max_launch_partial_columns", ctypes.c_int64)]


EXPORTS = ("rg_abi_version", "rg_status_string", "rg_draft_verify_attention_workspace",
           "rg_draft_verify_attention", "rg_draft_verify_attention_plan", "rg_draft_verify_attention_check",
           "rg_attention_launches", "rg_verify_accept_workspace", "rg_verify_accept", "rg_draft_confidence_workspace",
           "rg_draft_confidence", "rg_verify_and_confidence_workspace", "rg_verify_and_confidence",
           "rg_verify_and_confidence_noalloc",
           "rg_multibranch_attention_workspace", "rg_multibranch_attention", "rg_plan_branches",
           "rg_match_branches", "rg_plan_block_sizes", "rg_kv4_append", "rg_kv4_read", "rg_kv4_attention_workspace",
           "rg_kv4_attention", "rg_attention_mass", "rg_kv4_attention_mass", "rg_evict_workspace", "rg_evict_tokens",
           "rg_kv4_evict_tokens", "rg_kv_append", "rg_kv8_append", "rg_kv8_read",
           "rg_window_attention_workspace", "rg_window_attention", "rg_kv8_attention_workspace", "rg_kv8_attention")

_LIB = None


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built (run `python -m paper_2609_34388_amd.build_lib`)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    sig = {
        "rg_abi_version": (I32, []),
        "rg_status_string": (ctypes.c_char_p, [I32]),
        "rg_draft_verify_attention_workspace": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(SZ)]),
        "rg_draft_verify_attention_plan": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(AttnPlanInfo)]),
        "rg_attention_launches": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                        ctypes.POINTER(AttnLaunchInfo)]),
        "rg_draft_verify_attention": (I32, [ctypes.POINTER(AttnLayout), P, P, P, P, P, P, SZ, P]),
        "rg_draft_verify_attention_check": (I32, [P, SZ, P]),
        "rg_verify_accept_workspace": (I32, [I32, I32, I32, ctypes.POINTER(SZ)]),
        "rg_verify_accept": (I32, [P, I64, I32, I32, I32, P, P, P, P, P, P, P, P, SZ, P]),
        "rg_draft_confidence_workspace": (I32, [I32, I32, ctypes.POINTER(SZ)]),
        "rg_draft_confidence": (I32, [P, I64, I32, I32, P, P, P, P, P, P, P, SZ, P]),
        "rg_verify_and_confidence_workspace": (I32, [I32, I32, I32, I32, ctypes.POINTER(SZ)]),
        "rg_verify_and_confidence": (I32, [P, I64, P, I64, I32, I32, I32, P, P, P, P, P, P, P,
                                           I32, P, P, P, P, P, P, P, SZ, P]),
        "rg_verify_and_confidence_noalloc": (I32, [P, I64, P, I64, I32, I32, I32, P, P, P, P, P, P, P,
                                                   I32, P, P, P, P, P, P, P]),
        "rg_multibranch_attention_workspace": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                                     ctypes.POINTER(SZ)]),
        "rg_multibranch_attention": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                           P, P, P, P, P, P, SZ, P]),
        "rg_plan_branches": (I32, [P, P, P, I32, I32, ctypes.c_float, P, P, P, P, P, P]),
        "rg_match_branches": (I32, [P, P, P, P, P, P, P, P, I32, P, P]),
        "rg_plan_block_sizes": (I32, [ctypes.POINTER(BlockPolicy), P, P, P, P, I32, P, P, P, P]),
        "rg_kv4_append": (I32, [ctypes.POINTER(AttnLayout), P, I64, P, I64, P, P]),
        "rg_kv4_read": (I32, [ctypes.POINTER(AttnLayout), P, P, I64, P, I64, P]),
        "rg_kv4_attention_workspace": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                             ctypes.POINTER(SZ)]),
        "rg_kv4_attention": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout), P, P, P, P, P, SZ, P]),
        "rg_attention_mass": (I32, [ctypes.POINTER(AttnLayout), P, P, P, P, ctypes.c_float, P, P]),
        "rg_kv4_attention_mass": (I32, [ctypes.POINTER(AttnLayout), P, P, P, P, ctypes.c_float, P, P]),
        "rg_evict_workspace": (I32, [ctypes.POINTER(EvictLayout), ctypes.POINTER(SZ)]),
        "rg_evict_tokens": (I32, [ctypes.POINTER(EvictLayout), P, P, P, P, P, P, SZ, P]),
        "rg_kv4_evict_tokens": (I32, [ctypes.POINTER(EvictLayout), P, P, P, P, P, SZ, P]),
        "rg_kv_append": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(Rotation), P, I64, P, P, I64, P, I64, P, P, P]),
        "rg_kv8_append": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(Rotation), P, I64, P, P, I64, P, I64, P, P, P]),
        "rg_kv8_read": (I32, [ctypes.POINTER(AttnLayout), P, P, P, I64, P, I64, P]),
        "rg_window_attention_workspace": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                                ctypes.POINTER(Window), ctypes.POINTER(SZ)]),
        "rg_window_attention": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout), ctypes.POINTER(Window),
                                      P, P, P, P, P, P, SZ, P]),
        "rg_kv8_attention_workspace": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout),
                                             ctypes.POINTER(Window), ctypes.POINTER(SZ)]),
        "rg_kv8_attention": (I32, [ctypes.POINTER(AttnLayout), ctypes.POINTER(BranchLayout), ctypes.POINTER(Window),
                                   P, P, P, P, P, P, SZ, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def library() -> ctypes.CDLL:
    """The loaded library (raises if it is not built)."""
    return _lib()


def abi_version() -> int:
    return int(_lib().rg_abi_version())


# ---------------------------------------------------------------------------
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


def _dev(t: torch.Tensor, name: str, dtype: torch.dtype) -> torch.Tensor:
    if type(t) is torch.Tensor and t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _host_i32(x, name: str) -> np.ndarray:
    if isinstance(x, torch.Tensor):
        if x.is_cuda:
            raise TypeError(f"{name} must be a host array")
        x = x.numpy()
    a = np.ascontiguousarray(np.asarray(x), dtype=np.int32)
    return a


# The current stream's raw handle without building a torch.cuda.Stream around
# it (2.7 us of a call's 8 to 27): where this torch has the function.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _outputs(given: Optional[Dict[str, torch.Tensor]], device, *wanted) -> Dict[str, torch.Tensor]:
    """The caller's outputs, and a new tensor for each (name, size, dtype)
    of `wanted` that is not among them."""
    o = dict(given or {})
    for name, size, dtype in wanted:
        if name not in o:
            o[name] = torch.empty(size, dtype=dtype, device=device)
    return o


def _check(status: int, where: str):
    if status != RG_OK:
        raise RGError(status, where)


class _Layout:
    """Keeps the host arrays alive while the C struct points at them."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, num_pages, q_indptr, n_verify,
                 ctx_len, page_indptr, page_indices: torch.Tensor, sm_scale=0.0):
        self.q_indptr = _host_i32(q_indptr, "q_indptr")
        self.n_verify = _host_i32(n_verify, "n_verify")
        self.ctx_len = _host_i32(ctx_len, "ctx_len")
        self.page_indptr = _host_i32(page_indptr, "page_indptr")
        self.page_indices = _dev(page_indices, "page_indices", torch.int32)
        R = self.ctx_len.shape[0]
        if self.q_indptr.shape[0] != R + 1 or self.page_indptr.shape[0] != R + 1 or \
                self.n_verify.shape[0] != R:
            raise ValueError("per-request arrays disagree on the number of requests")
        self.c = AttnLayout(R, num_q_heads, num_kv_heads, head_dim, 16, num_pages, float(sm_scale),
                            self.q_indptr.ctypes.data, self.n_verify.ctypes.data,
                            self.ctx_len.ctypes.data, self.page_indptr.ctypes.data,
                            self.page_indices.data_ptr())
        # what calls ask for every time, without going through the struct
        self.ref = ctypes.byref(self.c)
        self.heads = (num_q_heads, num_kv_heads, head_dim)
        self.pools = {"k": (num_pages, num_kv_heads, 16, head_dim), "v": (num_pages, num_kv_heads, head_dim, 16),
                      "kv8": (num_pages, num_kv_heads, 32 * head_dim), "scales": (num_pages, num_kv_heads, 2)}


def make_layout(q: torch.Tensor, k_cache: torch.Tensor, q_indptr, n_verify, ctx_len, page_indptr,
                page_indices: torch.Tensor, sm_scale: float = 0.0) -> _Layout:
    total, hq, d = q.shape
    num_pages, hkv, page, d2 = k_cache.shape
    if page != 16 or d2 != d:
        raise ValueError("k_cache must be [pages, Hkv, 16, D] with the query's D")
    return _Layout(hq, hkv, d, num_pages, q_indptr, n_verify, ctx_len, page_indptr, page_indices,
                   sm_scale)


def attention_workspace_bytes(layout: _Layout) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_draft_verify_attention_workspace(ctypes.byref(layout.c), ctypes.byref(n)),
           "rg_draft_verify_attention_workspace")
    return int(n.value)


def attention_plan(layout: _Layout) -> Dict[str, int]:
    info = AttnPlanInfo()
    _check(_lib().rg_draft_verify_attention_plan(ctypes.byref(layout.c), ctypes.byref(info)),
           "rg_draft_verify_attention_plan")
    return {f: int(getattr(info, f)) for f, _ in AttnPlanInfo._fields_}


def attention_launches(layout: _Layout, branches: Optional["_Branches"] = None) -> Dict[str, int]:
    """What draft_verify_attention (or, with branches, multibranch_attention)
    launches for this layout."""
    info = AttnLaunchInfo()
    _check(_lib().rg_attention_launches(ctypes.byref(layout.c), ctypes.byref(branches.c) if branches else None,
                                        ctypes.byref(info)), "rg_attention_launches")
    return {f: int(getattr(info, f)) for f, _ in AttnLaunchInfo._fields_ if f != "reserved"}


def draft_verify_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                           q_indptr, n_verify, ctx_len, page_indptr, page_indices: torch.Tensor, *,
                           sm_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                           workspace: Optional[torch.Tensor] = None, layout: Optional[_Layout] = None,
                           stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Fused draft-verify attention (rg_draft_verify_attention).

    q [sum n, Hq, D], k_cache [pages, Hkv, 16, D], v_cache [pages, Hkv, D, 16]
    (bf16); returns (out [sum n, Hq, D] bf16, lse [sum n, Hq] fp32 or None).
    """
    _dev(q, "q", torch.bfloat16)
    _dev(k_cache, "k_cache", torch.bfloat16)
    _dev(v_cache, "v_cache", torch.bfloat16)
    if v_cache.shape != (k_cache.shape[0], k_cache.shape[1], k_cache.shape[3], 16):
        raise ValueError("v_cache must be [pages, Hkv, D, 16]")
    lay = layout or make_layout(q, k_cache, q_indptr, n_verify, ctx_len, page_indptr, page_indices, sm_scale)
    if int(lay.q_indptr[-1]) != q.shape[0]:
        raise ValueError("q_indptr[-1] must equal the number of query rows")
    if lay.page_indices.numel() < int(lay.page_indptr[-1]):
        raise ValueError("page_indices is shorter than page_indptr[-1]")
    if out is None:
        out = torch.empty_like(q)
    _dev(out, "out", torch.bfloat16)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[0], q.shape[1], dtype=torch.float32, device=q.device)
    if lse is not None:
        _dev(lse, "lse", torch.float32)
    if workspace is None:  # the call itself checks the size of one that is given
        need = attention_workspace_bytes(lay)
        if need:
            workspace = new_workspace(need, q.device)
    ws_ptr = _ptr(workspace) if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = _lib().rg_draft_verify_attention(ctypes.byref(lay.c), q.data_ptr(), k_cache.data_ptr(),
                                          v_cache.data_ptr(), out.data_ptr(), _ptr(lse), ws_ptr,
                                          ws_bytes, _stream(stream))
    _check(st, "rg_draft_verify_attention")
    return out, lse


def attention_check(workspace: torch.Tensor, stream=None) -> int:
    """rg_draft_verify_attention_check: synchronises the stream and returns
    the status (RG_OK, or 6 = RG_ERR_WAIT when a one-launch wait gave up)."""
    return int(_lib().rg_draft_verify_attention_check(workspace.data_ptr(), workspace.numel(), _stream(stream)))


class _Branches:
    """Host arrays of the overlap branches, kept alive with the C struct."""

    def __init__(self, branch_indptr, prefix, lead, rows):
        self.branch_indptr = _host_i32(branch_indptr, "branch_indptr")
        self.prefix = _host_i32(prefix, "prefix")
        self.lead = _host_i32(lead, "lead")
        self.rows = _host_i32(rows, "rows")
        nb = int(self.branch_indptr[-1]) if self.branch_indptr.size else 0
        for name in ("prefix", "lead", "rows"):
            if getattr(self, name).shape[0] < nb:
                raise ValueError(f"{name} is shorter than branch_indptr[-1]")
        self.c = BranchLayout(self.branch_indptr.ctypes.data, self.prefix.ctypes.data,
                              self.lead.ctypes.data, self.rows.ctypes.data)


def make_branches(branch_indptr, prefix, lead, rows) -> _Branches:
    return _Branches(branch_indptr, prefix, lead, rows)


def multibranch_workspace_bytes(layout: _Layout, branches: _Branches) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_multibranch_attention_workspace(ctypes.byref(layout.c), ctypes.byref(branches.c),
                                                     ctypes.byref(n)), "rg_multibranch_attention_workspace")
    return int(n.value)


def multibranch_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, layout: _Layout,
                          branches: _Branches, *, out: Optional[torch.Tensor] = None,
                          lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                          workspace: Optional[torch.Tensor] = None,
                          stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of a step with overlap branches (rg_multibranch_attention);
    tensors as in draft_verify_attention, the layout from make_layout and
    the branch lists from make_branches."""
    _dev(q, "q", torch.bfloat16)
    _dev(k_cache, "k_cache", torch.bfloat16)
    _dev(v_cache, "v_cache", torch.bfloat16)
    if v_cache.shape != (k_cache.shape[0], k_cache.shape[1], k_cache.shape[3], 16):
        raise ValueError("v_cache must be [pages, Hkv, D, 16]")
    if int(layout.q_indptr[-1]) != q.shape[0]:
        raise ValueError("q_indptr[-1] must equal the number of query rows")
    if branches.branch_indptr.shape[0] != layout.ctx_len.shape[0] + 1:
        raise ValueError("branch_indptr must have num_requests + 1 entries")
    if out is None:
        out = torch.empty_like(q)
    _dev(out, "out", torch.bfloat16)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[0], q.shape[1], dtype=torch.float32, device=q.device)
    if lse is not None:
        _dev(lse, "lse", torch.float32)
    if workspace is None:  # the call itself checks the size of one that is given
        need = multibranch_workspace_bytes(layout, branches)
        if need:
            workspace = new_workspace(need, q.device)
    ws_ptr = _ptr(workspace) if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = _lib().rg_multibranch_attention(ctypes.byref(layout.c), ctypes.byref(branches.c), q.data_ptr(),
                                         k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr(), _ptr(lse),
                                         ws_ptr, ws_bytes, _stream(stream))
    _check(st, "rg_multibranch_attention")
    return out, lse


def plan_branches(margin: torch.Tensor, top2: torch.Tensor, row_indptr: torch.Tensor, delta: float, *,
                  out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Risky positions and branches of each request's draft block
    (rg_plan_branches); margin fp32 / top2 int32 per draft row, row_indptr
    int32 [R+1] on the device."""
    _dev(margin, "margin", torch.float32)
    _dev(top2, "top2", torch.int32)
    _dev(row_indptr, "row_indptr", torch.int32)
    R = row_indptr.numel() - 1
    dev = margin.device
    if out is None:
        out = dict(n_risky=torch.empty(R, dtype=torch.int32, device=dev),
                   n_corr=torch.empty(R, dtype=torch.int32, device=dev),
                   corr_pos=torch.empty(R, 2, dtype=torch.int32, device=dev),
                   corr_tok=torch.empty(R, 2, dtype=torch.int32, device=dev),
                   continuation=torch.empty(R, dtype=torch.int32, device=dev))
    st = _lib().rg_plan_branches(_ptr(margin), _ptr(top2), row_indptr.data_ptr(), R, margin.numel(),
                                 ctypes.c_float(delta), out["n_risky"].data_ptr(), out["n_corr"].data_ptr(),
                                 out["corr_pos"].data_ptr(), out["corr_tok"].data_ptr(),
                                 out["continuation"].data_ptr(), _stream(stream))
    _check(st, "rg_plan_branches")
    return out


def match_branches(accept_len: torch.Tensor, next_token: torch.Tensor, block_len: torch.Tensor,
                   plan: Dict[str, torch.Tensor], cont_first: torch.Tensor, *,
                   out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Index of the branch each request's verification confirms, or -1
    (rg_match_branches); all int32 device tensors, `plan` from plan_branches."""
    for name, t in (("accept_len", accept_len), ("next_token", next_token), ("block_len", block_len),
                    ("cont_first", cont_first)):
        _dev(t, name, torch.int32)
    R = accept_len.numel()
    if out is None:
        out = torch.empty(R, dtype=torch.int32, device=accept_len.device)
    st = _lib().rg_match_branches(accept_len.data_ptr(), next_token.data_ptr(), block_len.data_ptr(),
                                  plan["n_corr"].data_ptr(), plan["corr_pos"].data_ptr(),
                                  plan["corr_tok"].data_ptr(), plan["continuation"].data_ptr(),
                                  cont_first.data_ptr(), R, out.data_ptr(), _stream(stream))
    _check(st, "rg_match_branches")
    return out


class _BlockPolicy:
    """An rg_block_policy with its host arrays kept alive."""

    def __init__(self, candidates, s_edges, cost, rho: float, value: torch.Tensor):
        self.candidates = np.ascontiguousarray(np.asarray(candidates), dtype=np.int32)
        self.s_edges = np.ascontiguousarray(np.asarray(s_edges, dtype=np.float32).reshape(-1))
        self.cost = np.ascontiguousarray(np.asarray(cost, dtype=np.float32).reshape(-1))
        _dev(value, "value", torch.float32)
        nb, ns = self.candidates.shape[0], self.s_edges.shape[0] + 1
        if tuple(value.shape) != (nb, ns, nb, 2):
            raise ValueError(f"value must be [{nb}, {ns}, {nb}, 2], got {tuple(value.shape)}")
        if self.cost.shape[0] != nb:
            raise ValueError("cost needs one entry per candidate")
        self.value = value
        self.c = BlockPolicy(nb, self.candidates.ctypes.data, ns,
                             self.s_edges.ctypes.data if ns > 1 else None, self.cost.ctypes.data,
                             float(rho), value.data_ptr())


def make_block_policy(candidates, s_edges, cost, rho: float, value: torch.Tensor) -> _BlockPolicy:
    """Policy of Eq. 3 at one load: candidate block sizes, s-bin edges, cost
    T_C(B) per candidate (host), rho_C, and the V_B table on the device as an
    fp32 tensor [NB, NS, NB, 2]."""
    return _BlockPolicy(candidates, s_edges, cost, rho, value)


def plan_block_sizes(policy: _BlockPolicy, accept_len: torch.Tensor, accept_entropy: torch.Tensor,
                     prev_block: torch.Tensor, entropy_hist: torch.Tensor, *, bucket: bool = True,
                     out: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Next block size per request and the grouping by size
    (rg_plan_block_sizes); entropy_hist is updated in place."""
    _dev(accept_len, "accept_len", torch.int32)
    _dev(accept_entropy, "accept_entropy", torch.float32)
    _dev(prev_block, "prev_block", torch.int32)
    _dev(entropy_hist, "entropy_hist", torch.float32)
    R = accept_len.numel()
    for name, t in (("accept_entropy", accept_entropy), ("prev_block", prev_block), ("entropy_hist", entropy_hist)):
        if t.numel() != R:
            raise ValueError(f"{name} must have {R} entries")
    dev = accept_len.device
    nb = policy.candidates.shape[0]
    if out is None:
        out = dict(next_block=torch.empty(R, dtype=torch.int32, device=dev))
        if bucket:
            out["order"] = torch.empty(R, dtype=torch.int32, device=dev)
            out["bucket_offsets"] = torch.empty(nb + 1, dtype=torch.int32, device=dev)
    st = _lib().rg_plan_block_sizes(ctypes.byref(policy.c), _ptr(accept_len), _ptr(accept_entropy),
                                    _ptr(prev_block), _ptr(entropy_hist), R, _ptr(out["next_block"]),
                                    _ptr(out.get("order")), _ptr(out.get("bucket_offsets")), _stream(stream))
    _check(st, "rg_plan_block_sizes")
    return out


def verify_accept_workspace_bytes(num_requests: int, total_rows: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_verify_accept_workspace(num_requests, total_rows, vocab, ctypes.byref(n)),
           "rg_verify_accept_workspace")
    return int(n.value)


def draft_confidence_workspace_bytes(total_rows: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_draft_confidence_workspace(total_rows, vocab, ctypes.byref(n)),
           "rg_draft_confidence_workspace")
    return int(n.value)


def new_workspace(nbytes: int, device) -> torch.Tensor:
    """A zeroed workspace of at least `nbytes` bytes.  Attention workspaces must be
    zero before their first use (each call leaves them ready for the next); the
    others need no initialisation."""
    return torch.zeros(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def verify_accept(logits: torch.Tensor, row_indptr: torch.Tensor, draft_tokens: torch.Tensor, *,
                  workspace: Optional[torch.Tensor] = None, out: Optional[Dict[str, torch.Tensor]] = None,
                  want_entropy: bool = True, stream=None) -> Dict[str, torch.Tensor]:
    """Greedy verification (rg_verify_accept).  logits [rows, vocab] bf16
    (row stride may exceed vocab), row_indptr [R+1] int32, draft_tokens
    [rows] int32 -- all on the GPU."""
    if not logits.is_cuda or logits.dtype != torch.bfloat16 or logits.dim() != 2 or logits.stride(1) != 1:
        raise TypeError("logits must be a CUDA bf16 [rows, vocab] tensor with unit column stride")
    _dev(row_indptr, "row_indptr", torch.int32)
    rows, vocab = logits.shape
    R = row_indptr.shape[0] - 1
    if rows:
        _dev(draft_tokens, "draft_tokens", torch.int32)
    dev = logits.device
    i, f = torch.int32, torch.float32
    o = _outputs(out, dev, ("row_argmax", rows, i), ("accept_len", R, i), ("next_token", R, i))
    if want_entropy:
        o = _outputs(o, dev, ("row_entropy", rows, f), ("accept_entropy", R, f))
    if workspace is None:
        workspace = new_workspace(verify_accept_workspace_bytes(R, rows, vocab), dev)
    st = _lib().rg_verify_accept(
        logits.data_ptr() if rows else None, logits.stride(0) if rows else vocab, vocab, R, rows,
        row_indptr.data_ptr(), draft_tokens.data_ptr() if rows else None,
        o["row_argmax"].data_ptr() if rows else None, o["accept_len"].data_ptr(),
        o["next_token"].data_ptr(), _ptr(o.get("row_entropy")) if rows else None,
        _ptr(o.get("accept_entropy")), workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(st, "rg_verify_accept")
    return o


def draft_confidence(logits: torch.Tensor, *, workspace: Optional[torch.Tensor] = None,
                     out: Optional[Dict[str, torch.Tensor]] = None, want_margin: bool = True,
                     want_entropy: bool = True, stream=None) -> Dict[str, torch.Tensor]:
    """Draft confidence (rg_draft_confidence) of logits [rows, vocab] bf16."""
    if not logits.is_cuda or logits.dtype != torch.bfloat16 or logits.dim() != 2 or logits.stride(1) != 1:
        raise TypeError("logits must be a CUDA bf16 [rows, vocab] tensor with unit column stride")
    rows, vocab = logits.shape
    dev = logits.device
    i, f = torch.int32, torch.float32
    o = _outputs(out, dev, ("top1", rows, i), ("top2", rows, i), ("p1", rows, f), ("p2", rows, f))
    if want_margin:
        o = _outputs(o, dev, ("margin", rows, f))
    if want_entropy:
        o = _outputs(o, dev, ("entropy", rows, f))
    if workspace is None:
        workspace = new_workspace(draft_confidence_workspace_bytes(rows, vocab), dev)
    st = _lib().rg_draft_confidence(
        logits.data_ptr() if rows else None, logits.stride(0) if rows else vocab, vocab, rows,
        _ptr(o["top1"]), _ptr(o["top2"]), _ptr(o["p1"]), _ptr(o["p2"]), _ptr(o.get("margin")),
        _ptr(o.get("entropy")), workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(st, "rg_draft_confidence")
    return o


def verify_and_confidence_workspace_bytes(num_requests: int, verify_rows: int, draft_rows: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_verify_and_confidence_workspace(num_requests, verify_rows, draft_rows, vocab, ctypes.byref(n)),
           "rg_verify_and_confidence_workspace")
    return int(n.value)


def verify_and_confidence(verify_logits: torch.Tensor, row_indptr: torch.Tensor, draft_tokens: torch.Tensor,
                          draft_logits: torch.Tensor, *, workspace: Optional[torch.Tensor] = None,
                          out_verify: Optional[Dict[str, torch.Tensor]] = None,
                          out_draft: Optional[Dict[str, torch.Tensor]] = None, noalloc: bool = False,
                          stream=None) -> Tuple[Dict[str, torch.Tensor], Dict[str, torch.Tensor]]:
    """Both logit passes of a round in one call (rg_verify_and_confidence):
    returns the outputs of verify_accept and of draft_confidence.  With
    ``noalloc`` the allocation-free variant runs instead
    (rg_verify_and_confidence_noalloc: the library's static scratch, no
    workspace; ``workspace`` is ignored)."""
    for t, name in ((verify_logits, "verify_logits"), (draft_logits, "draft_logits")):
        if not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != 2 or t.stride(1) != 1:
            raise TypeError(f"{name} must be a CUDA bf16 [rows, vocab] tensor with unit column stride")
    if verify_logits.shape[1] != draft_logits.shape[1]:
        raise ValueError("verify and draft logits must have the same vocabulary")
    _dev(row_indptr, "row_indptr", torch.int32)
    vrows, vocab = verify_logits.shape
    drows = draft_logits.shape[0]
    R = row_indptr.shape[0] - 1
    if vrows:
        _dev(draft_tokens, "draft_tokens", torch.int32)
    dev = verify_logits.device
    i, f = torch.int32, torch.float32
    ov = _outputs(out_verify, dev, ("row_argmax", vrows, i), ("accept_len", R, i), ("next_token", R, i),
                  ("row_entropy", vrows, f), ("accept_entropy", R, f))
    od = _outputs(out_draft, dev, ("top1", drows, i), ("top2", drows, i), ("p1", drows, f), ("p2", drows, f),
                  ("margin", drows, f), ("entropy", drows, f))
    args = (verify_logits.data_ptr() if vrows else None, verify_logits.stride(0) if vrows else vocab,
            draft_logits.data_ptr() if drows else None, draft_logits.stride(0) if drows else vocab, vocab, R, vrows,
            row_indptr.data_ptr(), draft_tokens.data_ptr() if vrows else None,
            ov["row_argmax"].data_ptr() if vrows else None, ov["accept_len"].data_ptr(), ov["next_token"].data_ptr(),
            _ptr(ov.get("row_entropy")) if vrows else None, _ptr(ov.get("accept_entropy")), drows,
            _ptr(od["top1"]) if drows else None, _ptr(od["top2"]) if drows else None,
            _ptr(od["p1"]) if drows else None, _ptr(od["p2"]) if drows else None,
            _ptr(od.get("margin")) if drows else None, _ptr(od.get("entropy")) if drows else None)
    if noalloc:
        _check(_lib().rg_verify_and_confidence_noalloc(*args, _stream(stream)), "rg_verify_and_confidence_noalloc")
        return ov, od
    if workspace is None:
        workspace = new_workspace(verify_and_confidence_workspace_bytes(R, vrows, drows, vocab), dev)
    st = _lib().rg_verify_and_confidence(*args, workspace.data_ptr(), workspace.numel(), _stream(stream))
    _check(st, "rg_verify_and_confidence")
    return ov, od



# ---------------------------------------------------------------------------
# A paged KV cache in 4 bits
def kv4_block_bytes(head_dim: int) -> int:
    """Bytes of K and V of 16 tokens of one KV head (RG_KV4_BLOCK_BYTES)."""
    return 17 * head_dim


def new_kv4_cache(num_pages: int, num_kv_heads: int, head_dim: int, device) -> torch.Tensor:
    """A 4-bit cache pool, uint8 [pages, Hkv, 17 D] (contents undefined)."""
    return torch.empty(num_pages, num_kv_heads, kv4_block_bytes(head_dim), dtype=torch.uint8, device=device)


def _kv4(cache: torch.Tensor, head_dim: int, num_kv_heads: int, num_pages: int) -> torch.Tensor:
    _dev(cache, "cache", torch.uint8)
    if cache.shape != (num_pages, num_kv_heads, 17 * head_dim):
        raise ValueError("cache must be [pages, Hkv, 17 D] of the layout's sizes")
    return cache


def make_kv4_layout(num_q_heads: int, cache: torch.Tensor, q_indptr, n_verify, ctx_len, page_indptr,
                    page_indices: torch.Tensor, sm_scale: float = 0.0) -> _Layout:
    """make_layout for a 4-bit cache (uint8 [pages, Hkv, 17 D])."""
    num_pages, hkv, block = cache.shape
    if block % 17:
        raise ValueError("cache must be [pages, Hkv, 17 D]")
    return _Layout(num_q_heads, hkv, block // 17, num_pages, q_indptr, n_verify, ctx_len, page_indptr, page_indices,
                   sm_scale)


# The current device without torch.cuda's own checks (0.6 us a call): tensors of
# a device are there, so it is initialised.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _here(*tensors: Optional[torch.Tensor]) -> int:
    """The current device, where a call's kernels run and its tensors have to be."""
    here = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor is on device {t.get_device()}, the current device is {here}")
    return here


def _check_layout(lay, rows: int, *tensors: Optional[torch.Tensor]) -> int:
    """Checks the arrays' lengths and the tensors' device; returns the device."""
    if lay.q_indptr.item(-1) != rows:
        raise ValueError("q_indptr[-1] must equal the number of rows")
    if lay.page_indices.numel() < lay.page_indptr.item(-1):
        raise ValueError("page_indices is shorter than page_indptr[-1]")
    return _here(lay.page_indices, *tensors)


def _pool_of(stream):
    """Where a call's own tensors come from: the memory pool of the stream that
    uses them, not of one that may still have work on the same memory, or give it
    away before the call has run."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        # 0 is the default stream's handle; ExternalStream(0) would be some other stream
        stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _rows(t: torch.Tensor, name: str, hkv: int, d: int) -> int:
    """Checks rows [rows, Hkv, D] (any row stride, heads contiguous) and returns the stride."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not torch.bfloat16:
        raise TypeError(f"{name} must be a CUDA bf16 tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} must have three dimensions")
    (rows, heads, width), (ahead, apart, next_to) = t.shape, t.stride()
    if heads != hkv or width != d or next_to != 1 or (hkv > 1 and apart != d):
        raise ValueError(f"{name} must be [rows, {hkv}, {d}], contiguous within a row")
    return ahead if rows > 1 else hkv * d


def _rows_call(name: str, k: torch.Tensor, v: torch.Tensor, cache: torch.Tensor, layout: _Layout, stream, out: str):
    """Checks and calls rg_kv4_append or rg_kv4_read."""
    c = layout.c
    hkv, d = c.num_kv_heads, c.head_dim
    ks, vs = _rows(k, "k" + out, hkv, d), _rows(v, "v" + out, hkv, d)
    _kv4(cache, d, hkv, c.num_pages)
    rows = k.shape[0]
    if v.shape[0] != rows:
        raise ValueError("k and v must have as many rows")
    here = _check_layout(layout, rows, k, v, cache)
    if rows == 0:
        return
    on = _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)
    ref, kp, vp, cp = ctypes.byref(c), k.data_ptr(), v.data_ptr(), cache.data_ptr()
    if out:
        status = _lib().rg_kv4_read(ref, cp, kp, ks, vp, vs, on)
    else:
        status = _lib().rg_kv4_append(ref, kp, ks, vp, vs, cp, on)
    _check(status, name)


def kv4_append(k: torch.Tensor, v: torch.Tensor, cache: torch.Tensor, layout: _Layout, *, stream=None) -> None:
    """Rows k, v [rows, Hkv, D] (e.g. parts of one projection's output) into
    the 4-bit cache, at the tokens behind each request's context
    (rg_kv4_append).  32 elements with an infinity or a NaN among them read as
    NaN."""
    _rows_call("rg_kv4_append", k, v, cache, layout, stream, "")


def kv4_read(cache: torch.Tensor, layout: _Layout, *, k_out: Optional[torch.Tensor] = None,
             v_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The tokens kv4_append writes for this layout, as bf16 rows (rg_kv4_read)."""
    k, v = k_out, v_out
    if k is None or v is None:
        _dev(cache, "cache", torch.uint8)
        shape = (int(layout.q_indptr[-1]), layout.c.num_kv_heads, layout.c.head_dim)
        with _pool_of(stream):
            k = torch.empty(shape, dtype=torch.bfloat16, device=cache.device) if k is None else k
            v = torch.empty(shape, dtype=torch.bfloat16, device=cache.device) if v is None else v
    _rows_call("rg_kv4_read", k, v, cache, layout, stream, "_out")
    return k, v


def kv4_attention_workspace_bytes(layout: _Layout, branches: Optional[_Branches] = None) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_kv4_attention_workspace(ctypes.byref(layout.c), ctypes.byref(branches.c) if branches else None,
                                             ctypes.byref(n)), "rg_kv4_attention_workspace")
    return int(n.value)


def kv4_attention(q: torch.Tensor, cache: torch.Tensor, layout: _Layout, branches: Optional[_Branches] = None, *,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                  workspace: Optional[torch.Tensor] = None,
                  stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """draft_verify_attention, or with branches multibranch_attention, over a
    4-bit cache (rg_kv4_attention); the layout from make_kv4_layout."""
    _dev(q, "q", torch.bfloat16)
    if q.dim() != 3 or q.shape[1] != layout.c.num_q_heads or q.shape[2] != layout.c.head_dim:
        raise ValueError("q must be [rows, Hq, D] of the layout's sizes")
    _kv4(cache, layout.c.head_dim, layout.c.num_kv_heads, layout.c.num_pages)
    _check_layout(layout, q.shape[0], q, cache, workspace)
    if branches is not None and branches.branch_indptr.shape[0] != layout.ctx_len.shape[0] + 1:
        raise ValueError("branch_indptr must have num_requests + 1 entries")
    if out is None or (lse is None and want_lse):
        with _pool_of(stream):
            out = torch.empty_like(q) if out is None else out
            if lse is None and want_lse:
                lse = torch.empty(q.shape[0], q.shape[1], dtype=torch.float32, device=q.device)
    if _dev(out, "out", torch.bfloat16).shape != q.shape:
        raise ValueError("out must have q's shape")
    if lse is not None and _dev(lse, "lse", torch.float32).shape != q.shape[:2]:
        raise ValueError("lse must be [rows, Hq]")
    _here(out, lse)
    if q.shape[0] == 0:
        return out, lse
    if workspace is None:  # the call itself checks the size of one that is given
        need = kv4_attention_workspace_bytes(layout, branches)
        if need:
            with _pool_of(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(_lib().rg_kv4_attention(ctypes.byref(layout.c), ctypes.byref(branches.c) if branches else None, q.data_ptr(),
                                   cache.data_ptr(), out.data_ptr(), _ptr(lse), _ptr(workspace), ws_bytes,
                                   _stream(stream)), "rg_kv4_attention")
    return out, lse


# ---------------------------------------------------------------------------
# Eviction of tokens by accumulated attention weight
def _slot_pool(t: torch.Tensor, name: str, dtype: torch.dtype, num_pages: int, num_kv_heads: int) -> torch.Tensor:
    if tuple(_dev(t, name, dtype).shape) != (num_pages, num_kv_heads, 16):
        raise ValueError(f"{name} must be [pages, Hkv, 16]")
    return t


def _mass_args(q, keys, lse, mass, layout: _Layout, row_count):
    _dev(q, "q", torch.bfloat16)
    if q.dim() != 3 or q.shape[1] != layout.c.num_q_heads or q.shape[2] != layout.c.head_dim:
        raise ValueError("q must be [rows, Hq, D] of the layout's sizes")
    if _dev(lse, "lse", torch.float32).shape != q.shape[:2]:
        raise ValueError("lse must be [rows, Hq]")
    _slot_pool(mass, "mass", torch.float32, layout.c.num_pages, layout.c.num_kv_heads)
    if row_count is not None and _dev(row_count, "row_count", torch.int32).numel() != layout.c.num_requests:
        raise ValueError("row_count needs one entry per request")
    _check_layout(layout, q.shape[0], q, keys, lse, mass, row_count)
    return lse.data_ptr(), _ptr(row_count)


def attention_mass(q: torch.Tensor, k_cache: torch.Tensor, lse: torch.Tensor, mass: torch.Tensor, layout: _Layout, *,
                   row_count: Optional[torch.Tensor] = None, decay: float = 1.0, stream=None) -> torch.Tensor:
    """Adds the verify rows' attention weights to the keys' mass (fp32
    [pages, Hkv, 16], in place; rg_attention_mass).  q, lse and the layout are
    those of the step's attention; row_count int32 [R]: the rows that count."""
    _dev(k_cache, "k_cache", torch.bfloat16)
    if tuple(k_cache.shape) != (layout.c.num_pages, layout.c.num_kv_heads, 16, layout.c.head_dim):
        raise ValueError("k_cache must be [pages, Hkv, 16, D] of the layout's sizes")
    lp, rp = _mass_args(q, k_cache, lse, mass, layout, row_count)
    if q.shape[0]:
        _check(_lib().rg_attention_mass(ctypes.byref(layout.c), q.data_ptr(), k_cache.data_ptr(), lp, rp, decay,
                                        mass.data_ptr(), _stream(stream)), "rg_attention_mass")
    return mass


def kv4_attention_mass(q: torch.Tensor, cache: torch.Tensor, lse: torch.Tensor, mass: torch.Tensor, layout: _Layout, *,
                       row_count: Optional[torch.Tensor] = None, decay: float = 1.0, stream=None) -> torch.Tensor:
    """attention_mass over a 4-bit cache (rg_kv4_attention_mass)."""
    _kv4(cache, layout.c.head_dim, layout.c.num_kv_heads, layout.c.num_pages)
    lp, rp = _mass_args(q, cache, lse, mass, layout, row_count)
    if q.shape[0]:
        _check(_lib().rg_kv4_attention_mass(ctypes.byref(layout.c), q.data_ptr(), cache.data_ptr(), lp, rp, decay,
                                            mass.data_ptr(), _stream(stream)), "rg_kv4_attention_mass")
    return mass


class _EvictLayout:
    """Keeps the host arrays alive while the C struct points at them."""

    def __init__(self, num_kv_heads, head_dim, num_pages, ctx_len, keep, tracked, evicted, page_indptr,
                 page_indices, sink, recent):
        self.ctx_len = _host_i32(ctx_len, "ctx_len")
        R = self.ctx_len.shape[0]
        zero = np.zeros(R, dtype=np.int32)
        self.keep = _host_i32(keep, "keep")
        self.tracked = zero if tracked is None else _host_i32(tracked, "tracked")
        self.evicted = zero if evicted is None else _host_i32(evicted, "evicted")
        self.page_indptr = _host_i32(page_indptr, "page_indptr")
        self.page_indices = _dev(page_indices, "page_indices", torch.int32)
        if any(a.shape != (R,) for a in (self.keep, self.tracked, self.evicted)) or self.page_indptr.shape != (R + 1,):
            raise ValueError("per-request arrays disagree on the number of requests")
        if self.page_indices.numel() < int(self.page_indptr[-1]):
            raise ValueError("page_indices is shorter than page_indptr[-1]")
        self.c = EvictLayout(R, num_kv_heads, head_dim, 16, num_pages, int(sink), int(recent), self.ctx_len.ctypes.data,
                             self.keep.ctypes.data, self.tracked.ctypes.data, self.evicted.ctypes.data,
                             self.page_indptr.ctypes.data, self.page_indices.data_ptr())


def make_evict_layout(cache: torch.Tensor, ctx_len, keep, page_indptr, page_indices: torch.Tensor, *, tracked=None,
                      evicted=None, sink: int = 0, recent: int = 0) -> _EvictLayout:
    """Requests to cut to `keep` tokens; cache is the bf16 K pool [pages, Hkv,
    16, D] or a 4-bit pool [pages, Hkv, 17 D].  tracked and evicted as an
    earlier call left them (None: zero)."""
    if cache.dim() == 3:
        if cache.shape[2] % 17:
            raise ValueError("cache must be [pages, Hkv, 17 D]")
        d = cache.shape[2] // 17
    elif cache.dim() == 4 and cache.shape[2] == 16:
        d = cache.shape[3]
    else:
        raise ValueError("cache must be a K pool [pages, Hkv, 16, D] or a 4-bit pool [pages, Hkv, 17 D]")
    return _EvictLayout(cache.shape[1], d, cache.shape[0], ctx_len, keep, tracked, evicted, page_indptr, page_indices,
                        sink, recent)


def evict_workspace_bytes(layout: _EvictLayout) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib().rg_evict_workspace(ctypes.byref(layout.c), ctypes.byref(n)), "rg_evict_workspace")
    return int(n.value)


def _evict_args(score, positions, layout: _EvictLayout, mass, workspace, stream):
    """The arguments behind the caches', and the workspace, which has to live until the call is made."""
    pool = (layout.c.num_pages, layout.c.num_kv_heads)
    _slot_pool(score, "score", torch.float32, *pool)
    _slot_pool(positions, "positions", torch.int32, *pool)
    if mass is not None:
        _slot_pool(mass, "mass", torch.float32, *pool)
    _here(score, positions, mass, workspace, layout.page_indices)
    if workspace is None:
        with _pool_of(stream):
            workspace = torch.empty(evict_workspace_bytes(layout), dtype=torch.uint8, device=score.device)
    return (score.data_ptr(), _ptr(mass), positions.data_ptr(), workspace.data_ptr(),
            workspace.numel() * workspace.element_size()), workspace


def evict_tokens(k_cache: torch.Tensor, v_cache: torch.Tensor, score: torch.Tensor, positions: torch.Tensor,
                 layout: _EvictLayout, *, mass: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Cuts each request to its best-scored tokens, in place
    (rg_evict_tokens): k_cache [pages, Hkv, 16, D], v_cache [pages, Hkv, D,
    16], score and mass fp32 and positions int32 [pages, Hkv, 16]."""
    c = layout.c
    _dev(k_cache, "k_cache", torch.bfloat16)
    _dev(v_cache, "v_cache", torch.bfloat16)
    if tuple(k_cache.shape) != (c.num_pages, c.num_kv_heads, 16, c.head_dim) or \
            tuple(v_cache.shape) != (c.num_pages, c.num_kv_heads, c.head_dim, 16):
        raise ValueError("k_cache must be [pages, Hkv, 16, D] and v_cache [pages, Hkv, D, 16] of the layout's sizes")
    _here(k_cache, v_cache)
    args, workspace = _evict_args(score, positions, layout, mass, workspace, stream)
    _check(_lib().rg_evict_tokens(ctypes.byref(c), k_cache.data_ptr(), v_cache.data_ptr(), *args, _stream(stream)),
           "rg_evict_tokens")


def kv4_evict_tokens(cache: torch.Tensor, score: torch.Tensor, positions: torch.Tensor, layout: _EvictLayout, *,
                     mass: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """evict_tokens on a 4-bit cache (rg_kv4_evict_tokens)."""
    c = layout.c
    _kv4(cache, c.head_dim, c.num_kv_heads, c.num_pages)
    _here(cache)
    args, workspace = _evict_args(score, positions, layout, mass, workspace, stream)
    _check(_lib().rg_kv4_evict_tokens(ctypes.byref(c), cache.data_ptr(), *args, _stream(stream)), "rg_kv4_evict_tokens")


# ---------------------------------------------------------------------------
# Rows into the cache with the rotation of their positions
class _Rotation:
    """Keeps the tensors alive while the C struct points at them."""

    def __init__(self, inv_freq, interleaved, positions):
        self.inv_freq = _dev(inv_freq, "inv_freq", torch.float32)
        self.positions = None if positions is None else _dev(positions, "positions", torch.int32)
        if inv_freq.dim() != 1 or (positions is not None and positions.dim() != 1):
            raise ValueError("inv_freq and positions must have one dimension")
        self.c = Rotation(2 * inv_freq.numel(), int(bool(interleaved)), inv_freq.data_ptr(), _ptr(positions))
        self.ref = ctypes.byref(self.c)


def make_rotation(inv_freq: torch.Tensor, *, interleaved: bool = False,
                  positions: Optional[torch.Tensor] = None) -> _Rotation:
    """The rotation of q and K rows (rg_rotation): inv_freq fp32 [dims / 2] on
    the GPU, positions int32 [rows] there (None: each row's token)."""
    return _Rotation(inv_freq, interleaved, positions)


def _append(name: str, k, v, caches, layout: _Layout, rotation: Optional[_Rotation], q, q_out, stream):
    """Checks and calls rg_kv_append or rg_kv8_append."""
    hq, hkv, d = layout.heads
    ks, vs, qs, qp, op = _rows(k, "k", hkv, d), _rows(v, "v", hkv, d), 0, None, None
    rows = k.shape[0]
    if v.shape[0] != rows:
        raise ValueError("k and v must have as many rows")
    if q is not None:
        qs = _rows(q, "q", hq, d)
        if q.shape[0] != rows:
            raise ValueError("q and k must have as many rows")
        if q_out is None:
            with _pool_of(stream):
                q_out = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=q.device)
        elif _dev(q_out, "q_out", torch.bfloat16).shape != q.shape:
            raise ValueError("q_out must have q's shape")
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out is given without q")
    ref = None
    here = _check_layout(layout, rows, k, v, q, q_out, *caches)
    if rotation is not None:
        if rotation.positions is not None and rotation.positions.shape[0] != rows:
            raise ValueError("positions needs one entry per row")
        _here(rotation.inv_freq, rotation.positions)
        ref = rotation.ref
    if rows:
        on = _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)
        _check(getattr(_lib(), name)(layout.ref, ref, qp, qs, op, k.data_ptr(), ks, v.data_ptr(), vs,
                                     caches[0].data_ptr(), caches[1].data_ptr(), on), name)
    return q_out


def _bf16_pools(k_cache: torch.Tensor, v_cache: torch.Tensor, layout: _Layout) -> None:
    if _dev(k_cache, "k_cache", torch.bfloat16).shape != layout.pools["k"]:
        raise ValueError("k_cache must be [pages, Hkv, 16, D] of the layout's sizes")
    if _dev(v_cache, "v_cache", torch.bfloat16).shape != layout.pools["v"]:
        raise ValueError("v_cache must be [pages, Hkv, D, 16] of the layout's sizes")


def kv_append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, layout: _Layout, *,
              rotation: Optional[_Rotation] = None, q: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Rows k, v [rows, Hkv, D] (e.g. parts of one projection's output) into the
    bf16 cache k_cache [pages, Hkv, 16, D], v_cache [pages, Hkv, D, 16], at the
    tokens behind each request's context, k turned by its rows' positions
    (rg_kv_append).  With q [rows, Hq, D], returns it turned."""
    _bf16_pools(k_cache, v_cache, layout)
    return _append("rg_kv_append", k, v, (k_cache, v_cache), layout, rotation, q, q_out, stream)


# ---------------------------------------------------------------------------
# A paged KV cache in 8 bits
def kv8_block_bytes(head_dim: int) -> int:
    """Bytes of K and V of 16 tokens of one KV head (RG_KV8_BLOCK_BYTES)."""
    return 32 * head_dim


def new_kv8_cache(num_pages: int, num_kv_heads: int, head_dim: int, device) -> Tuple[torch.Tensor, torch.Tensor]:
    """An 8-bit cache pool, uint8 [pages, Hkv, 32 D], and its scales, fp32
    [pages, Hkv, 2] (contents undefined)."""
    return (torch.empty(num_pages, num_kv_heads, kv8_block_bytes(head_dim), dtype=torch.uint8, device=device),
            torch.empty(num_pages, num_kv_heads, 2, dtype=torch.float32, device=device))


def make_kv8_layout(num_q_heads: int, cache: torch.Tensor, q_indptr, n_verify, ctx_len, page_indptr,
                    page_indices: torch.Tensor, sm_scale: float = 0.0) -> _Layout:
    """make_layout for an 8-bit cache (uint8 [pages, Hkv, 32 D])."""
    num_pages, hkv, block = cache.shape
    if block % 32:
        raise ValueError("cache must be [pages, Hkv, 32 D]")
    return _Layout(num_q_heads, hkv, block // 32, num_pages, q_indptr, n_verify, ctx_len, page_indptr, page_indices,
                   sm_scale)


def _kv8(cache: torch.Tensor, scales: torch.Tensor, layout: _Layout) -> None:
    if _dev(cache, "cache", torch.uint8).shape != layout.pools["kv8"]:
        raise ValueError("cache must be [pages, Hkv, 32 D] of the layout's sizes")
    if _dev(scales, "scales", torch.float32).shape != layout.pools["scales"]:
        raise ValueError("scales must be [pages, Hkv, 2] of the layout's sizes")


def kv8_append(k: torch.Tensor, v: torch.Tensor, cache: torch.Tensor, scales: torch.Tensor, layout: _Layout, *,
               rotation: Optional[_Rotation] = None, q: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """kv_append into the 8-bit cache (rg_kv8_append).  An infinity or a NaN
    reads as NaN."""
    _kv8(cache, scales, layout)
    return _append("rg_kv8_append", k, v, (cache, scales), layout, rotation, q, q_out, stream)


def kv8_read(cache: torch.Tensor, scales: torch.Tensor, layout: _Layout, *, k_out: Optional[torch.Tensor] = None,
             v_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The tokens kv8_append writes for this layout, as bf16 rows (rg_kv8_read)."""
    _kv8(cache, scales, layout)
    _, hkv, d = layout.heads
    if k_out is None or v_out is None:
        shape = (layout.q_indptr.item(-1), hkv, d)
        with _pool_of(stream):
            k_out = torch.empty(shape, dtype=torch.bfloat16, device=cache.device) if k_out is None else k_out
            v_out = torch.empty(shape, dtype=torch.bfloat16, device=cache.device) if v_out is None else v_out
    ks, vs = _rows(k_out, "k_out", hkv, d), _rows(v_out, "v_out", hkv, d)
    rows = k_out.shape[0]
    if v_out.shape[0] != rows:
        raise ValueError("k_out and v_out must have as many rows")
    here = _check_layout(layout, rows, k_out, v_out, cache, scales)
    if rows:
        on = _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)
        _check(_lib().rg_kv8_read(layout.ref, cache.data_ptr(), scales.data_ptr(), k_out.data_ptr(), ks,
                                  v_out.data_ptr(), vs, on), "rg_kv8_read")
    return k_out, v_out


# ---------------------------------------------------------------------------
# Attention over a sliding window with sinks, and over the 8-bit cache
def make_window(size: int, sink: int = 0) -> Window:
    """The latest `size` positions up to a row's own, and the first `sink` (rg_window)."""
    if max(abs(size), abs(sink)) >= 1 << 31:  # ctypes would cut it to 32 bits
        raise ValueError("a window's size and sinks are 32-bit numbers")
    return Window(int(size), int(sink))


def _window_args(layout: _Layout, branches: Optional[_Branches], window: Optional[Window]):
    if branches is not None and branches.branch_indptr.shape[0] != layout.ctx_len.shape[0] + 1:
        raise ValueError("branch_indptr must have num_requests + 1 entries")
    return (layout.ref, ctypes.byref(branches.c) if branches is not None else None,
            ctypes.byref(window) if window is not None else None)


def _window_workspace_bytes(name: str, layout, branches, window) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_lib(), name)(*_window_args(layout, branches, window), ctypes.byref(n)), name)
    return int(n.value)


def _window_call(name: str, q, caches, layout: _Layout, branches, window, out, lse, want_lse, workspace, stream):
    shape = _dev(q, "q", torch.bfloat16).shape
    if len(shape) != 3 or shape[1] != layout.heads[0] or shape[2] != layout.heads[2]:
        raise ValueError("q must be [rows, Hq, D] of the layout's sizes")
    rows = shape[0]
    if out is None or (lse is None and want_lse):
        with _pool_of(stream):
            out = torch.empty_like(q) if out is None else out
            if lse is None and want_lse:
                lse = torch.empty(rows, shape[1], dtype=torch.float32, device=q.device)
    if _dev(out, "out", torch.bfloat16).shape != shape:
        raise ValueError("out must have q's shape")
    if lse is not None and _dev(lse, "lse", torch.float32).shape != shape[:2]:
        raise ValueError("lse must be [rows, Hq]")
    here = _check_layout(layout, rows, q, out, lse, workspace, *caches)
    args = _window_args(layout, branches, window)
    if rows == 0:
        return out, lse
    if workspace is None:  # the call itself checks the size of one that is given
        need = _window_workspace_bytes(name + "_workspace", layout, branches, window)
        if need:
            with _pool_of(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    on = _raw_stream(here) if stream is None and _raw_stream is not None else _stream(stream)
    _check(getattr(_lib(), name)(*args, q.data_ptr(), *(t.data_ptr() for t in caches), out.data_ptr(), _ptr(lse),
                                 _ptr(workspace), ws_bytes, on), name)
    return out, lse


def window_attention_workspace_bytes(layout: _Layout, window: Window, branches: Optional[_Branches] = None) -> int:
    return _window_workspace_bytes("rg_window_attention_workspace", layout, branches, window)


def window_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, layout: _Layout, window: Window,
                     branches: Optional[_Branches] = None, *, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                     workspace: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """draft_verify_attention, or with branches multibranch_attention, over a
    sliding window with sinks (rg_window_attention)."""
    _bf16_pools(k_cache, v_cache, layout)
    return _window_call("rg_window_attention", q, (k_cache, v_cache), layout, branches, window, out, lse, want_lse,
                        workspace, stream)


def kv8_attention_workspace_bytes(layout: _Layout, branches: Optional[_Branches] = None, *,
                                  window: Optional[Window] = None) -> int:
    return _window_workspace_bytes("rg_kv8_attention_workspace", layout, branches, window)


def kv8_attention(q: torch.Tensor, cache: torch.Tensor, scales: torch.Tensor, layout: _Layout,
                  branches: Optional[_Branches] = None, *, window: Optional[Window] = None,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                  workspace: Optional[torch.Tensor] = None,
                  stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """draft_verify_attention, or with branches multibranch_attention, over an
    8-bit cache, over all keys or a window (rg_kv8_attention); the layout from
    make_kv8_layout."""
    _kv8(cache, scales, layout)
    return _window_call("rg_kv8_attention", q, (cache, scales), layout, branches, window, out, lse, want_lse, workspace,
                        stream)
