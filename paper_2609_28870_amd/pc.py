"""Thin ctypes binding of libpc (include/pc.h).

Argument marshalling only: every step of the hot path runs in the HIP
kernels of ``libpc.so``.  PyTorch provides device memory and the current HIP
stream.  Unsigned arrays travel in signed torch tensors of the same width
(uint64 bit patterns in int64, uint32 in int32); ``as_u64`` / ``as_u32``
reinterpret them on the host.

There is no fallback: if ``libpc.so`` is missing or no GPU is visible, calls
raise.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_lib", "libpc.so")
NONE = 0xFFFFFFFF
DEEPEST_FIRST = 1   # PC_HASH_DEEPEST_FIRST
PREV_ONLY = 2       # PC_PREV_ONLY
ROPE_INTERLEAVED, ROPE_TRANSPOSE = 1, 2   # PC_ROPE_INTERLEAVED, PC_ROPE_TRANSPOSE

_lib = None

_vp = ctypes.c_void_p
_u64 = ctypes.c_uint64
_u32 = ctypes.c_uint32
_sz = ctypes.c_size_t
_st = ctypes.c_int


class PcError(RuntimeError):
    pass


class _KvCache(ctypes.Structure):
    """pc_kv_cache"""
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("stride_page", _u64),
                ("stride_head", _u64), ("stride_slot", _u64), ("dtype", _u32), ("n_pages", _u32), ("page_size", _u32),
                ("n_kv_heads", _u32), ("head_dim", _u32)]


class _Rotation(ctypes.Structure):
    """pc_rotation"""
    _fields_ = [("table", _vp), ("pos", _vp), ("n_pos", _u32), ("rot_dim", _u32), ("flags", _u32)]


def lib():
    """Load libpc.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise PcError("libpc.so not built: run paper_2609_28870_amd/build.py (or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    L.pc_status_string.restype = ctypes.c_char_p
    L.pc_status_string.argtypes = [_st]
    L.pc_version.restype = ctypes.c_int
    L.pc_hash_blocks_ws.restype = _sz
    L.pc_hash_blocks_ws.argtypes = [_u32]
    L.pc_hash_blocks.restype = _st
    L.pc_hash_blocks.argtypes = [_vp, _u64, _vp, _vp, _u32, _u32, _vp, _u64, _vp, _u64, _vp, _vp,
                                 _vp, _u32, _vp, _sz, _vp]
    L.pc_prev_next_use_ws.restype = _sz
    L.pc_prev_next_use_ws.argtypes = [_u64]
    L.pc_prev_next_use.restype = _st
    L.pc_prev_next_use.argtypes = [_vp, _u64, _vp, _vp, _vp, _vp, _sz, _vp]
    L.pc_prev_next_chained_ws.restype = _sz
    L.pc_prev_next_chained_ws.argtypes = [_u64, _u32]
    L.pc_prev_next_chained.restype = _st
    L.pc_prev_next_chained.argtypes = [_vp, _u64, _vp, _u32, _u32, _vp, _vp, _vp, _vp, _sz, _vp]
    L.pc_stack_distance_runs_ws.restype = _sz
    L.pc_stack_distance_runs_ws.argtypes = [_u64]
    L.pc_stack_distance_runs.restype = _st
    L.pc_stack_distance_runs.argtypes = [_vp, _vp, _u64, _vp, _vp, _sz, _vp]
    L.pc_stack_distance_noalloc_max_n.restype = _u64
    L.pc_stack_distance_noalloc_max_n.argtypes = []
    L.pc_stack_distance_noalloc.restype = _st
    L.pc_stack_distance_noalloc.argtypes = [_vp, _vp, _u64, _vp, _vp]
    L.pc_stack_distance_ws.restype = _sz
    L.pc_stack_distance_ws.argtypes = [_u64]
    L.pc_stack_distance.restype = _st
    L.pc_stack_distance.argtypes = [_vp, _vp, _u64, _vp, _vp, _sz, _vp]
    L.pc_request_order_ws.restype = _sz
    L.pc_request_order_ws.argtypes = []
    L.pc_request_order.restype = _st
    L.pc_request_order.argtypes = [_vp, _vp, _vp, _u32, _u64, _vp, _vp, _vp, _sz, _vp]
    L.pc_stack_distance_req_ws.restype = _sz
    L.pc_stack_distance_req_ws.argtypes = []
    L.pc_stack_distance_req.restype = _st
    L.pc_stack_distance_req.argtypes = [_vp, _vp, _vp, _u32, _u64, _vp, _vp, _sz, _vp]
    L.pc_stack_distance_session_ws.restype = _sz
    L.pc_stack_distance_session_ws.argtypes = [_u64, _u32]
    L.pc_stack_distance_session.restype = _st
    L.pc_stack_distance_session.argtypes = [_vp, _vp, _vp, _u32, _u64, _vp, _vp, _sz, _vp]
    L.pc_reuse_profile_ws.restype = _sz
    L.pc_reuse_profile_ws.argtypes = [_u64]
    L.pc_reuse_profile.restype = _st
    L.pc_reuse_profile.argtypes = [_vp, _vp, _vp, _vp, _u32, _u64, _vp, _u32, _u32, _vp, _vp, _vp, _vp, _vp,
                                   _sz, _vp]
    L.pc_session_profile_ws.restype = _sz
    L.pc_session_profile_ws.argtypes = [_u32]
    L.pc_session_profile.restype = _st
    L.pc_session_profile.argtypes = [_vp, _vp, _vp, _u32, _u64, _vp, _u32, _u32, _u32, _vp, _vp, _vp, _vp, _vp,
                                     _sz, _vp]
    L.pc_mrc_weighted_ws.restype = _sz
    L.pc_mrc_weighted_ws.argtypes = [_u64, _u32]
    L.pc_mrc_weighted.restype = _st
    L.pc_mrc_weighted.argtypes = [_vp, _vp, _vp, _u64, _vp, _u32, _u64, _u64, _vp, _vp, _vp, _vp,
                                  _vp, _vp, _sz, _vp]
    L.pc_mrc_weighted_layout_ws.restype = _sz
    L.pc_mrc_weighted_layout_ws.argtypes = [_u64, _u32]
    L.pc_mrc_weighted_layout.restype = _st
    L.pc_mrc_weighted_layout.argtypes = [_vp, _vp, _u32, _u32, _vp, _u64, _vp, _u32, _u64, _u64, _vp, _vp, _vp,
                                         _vp, _vp, _vp, _sz, _vp]
    L.pc_belady_ws.restype = _sz
    L.pc_belady_ws.argtypes = [_u64, _u32]
    L.pc_belady.restype = _st
    L.pc_belady.argtypes = [_vp, _vp, _u64, _vp, _u32, _vp, _vp, _vp, _vp, _sz, _vp]
    L.pc_kv_append_ws.restype = _sz
    L.pc_kv_append_ws.argtypes = []
    L.pc_kv_append.restype = _st
    L.pc_kv_append.argtypes = [_vp, _vp, _u64, _vp, _vp, _u32, _u32, _u32, _vp, _u64, _u64, _vp, _u64, _u64, _u32,
                               _vp, _sz, _vp]
    L.pc_rope_table.restype = _st
    L.pc_rope_table.argtypes = [_vp, _u32, _u64, _u64, ctypes.c_double, _vp, _vp]
    L.pc_rope_ws.restype = _sz
    L.pc_rope_ws.argtypes = []
    L.pc_rope.restype = _st
    L.pc_rope.argtypes = [_vp, _vp, _u64, _u64, _vp, _u64, _u64, _u32, _u32, _u32, _u32, _vp, _sz, _vp]
    L.pc_kv_append_rope_ws.restype = _sz
    L.pc_kv_append_rope_ws.argtypes = []
    L.pc_kv_append_rope.restype = _st
    L.pc_kv_append_rope.argtypes = [_vp, _vp, _u64, _vp, _vp, _u32, _u32, _u32, _vp, _vp, _u64, _u64, _vp, _u64, _u64,
                                    _vp, _u64, _u64, _vp, _u64, _u64, _u32, _u32, _vp, _sz, _vp]
    L.pc_attn_paged_ws.restype = _sz
    L.pc_attn_paged_ws.argtypes = [_u32, _u32, _u32, _u32, _u32, _u32, _u32, ctypes.c_int]
    L.pc_attn_paged.restype = _st
    L.pc_attn_paged.argtypes = [_vp, _vp, _u64, _vp, _vp, _u32, _u32, _u32, _u32, _vp, _u64, _u64, _u32, _u32,
                                ctypes.c_float, _u32, _u32, _vp, _u64, _u64, _vp, _vp, _vp, _u64, _vp, _sz, _vp]
    L.pc_kv_evict_ws.restype = _sz
    L.pc_kv_evict_ws.argtypes = [_u32, _u32, _u32]
    L.pc_kv_evict.restype = _st
    L.pc_kv_evict.argtypes = [_vp, _vp, _u64, _vp, _u32, _u32, _vp, _u64, _u32, _u32, _vp, _u64, _vp, _vp, _vp, _vp,
                              _sz, _vp]
    L.pc_workspace_status.restype = _st
    L.pc_workspace_status.argtypes = [_vp, _sz, _vp, ctypes.POINTER(ctypes.c_int32)]
    L.pc_prof_enable.restype = None
    L.pc_prof_enable.argtypes = [ctypes.c_int]
    L.pc_prof_kernel_count.restype = ctypes.c_int
    L.pc_prof_kernel_name.restype = ctypes.c_char_p
    L.pc_prof_kernel_name.argtypes = [ctypes.c_int]
    L.pc_prof_read.restype = _st
    L.pc_prof_read.argtypes = [ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_double),
                               ctypes.c_int]
    _lib = L
    return L


def check(status: int) -> None:
    if status != 0:
        raise PcError("libpc: %s (%d)" % (lib().pc_status_string(status).decode(), status))


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise PcError("expected a GPU tensor")
    if not t.is_contiguous():
        raise PcError("expected a contiguous tensor")
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dev():
    if not torch.cuda.is_available():
        raise PcError("no GPU visible: libpc needs an MI355X (gfx950)")
    return torch.device("cuda", torch.cuda.current_device())


def workspace(nbytes: int) -> torch.Tensor:
    """Device scratch for one call (torch's allocator aligns to >= 256 B)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=_dev())


def workspace_status(ws: torch.Tensor) -> int:
    """Device-side status code of a workspace (synchronises the stream)."""
    code = ctypes.c_int32(0)
    check(lib().pc_workspace_status(_ptr(ws), ws.numel(), _stream(), ctypes.byref(code)))
    return int(code.value)


def as_u64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().numpy().view(np.uint64)


def as_u32(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().numpy().view(np.uint32)


def to_dev_u64(a) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint64).view(np.int64)).to(_dev())


def to_dev_u32(a) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint32).view(np.int32)).to(_dev())


# ------------------------------------------------------------------ stages

def hash_blocks(tokens: torch.Tensor, tok_start: torch.Tensor, tok_len: torch.Tensor,
                blk_off: torch.Tensor, n_blocks: int, block_size: int = 16,
                parent: Optional[torch.Tensor] = None, root: int = 0, want_depth: bool = True,
                keys: Optional[torch.Tensor] = None, depth: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, key_hist: Optional[torch.Tensor] = None,
                deepest_first: bool = False):
    """pc_hash_blocks: keys (int64 bits of uint64) and depth (int32 bits);
    with ``key_hist`` (int32[1024]) also the byte histograms of the keys'
    low four bytes, which prev_next_use can take instead of counting them.
    ``deepest_first`` writes each request's blocks in descending depth order
    (the recency order of request-level residency)."""
    L = lib()
    dev = _dev()
    n_seqs = tok_len.numel()
    if keys is None:
        keys = torch.empty(n_blocks, dtype=torch.int64, device=dev)
    if want_depth and depth is None:
        depth = torch.empty(n_blocks, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(L.pc_hash_blocks_ws(n_seqs))
    check(L.pc_hash_blocks(_ptr(tokens), tokens.numel(), _ptr(tok_start), _ptr(tok_len), n_seqs,
                           block_size, _ptr(parent), root & (2 ** 64 - 1), _ptr(blk_off), n_blocks,
                           _ptr(keys), _ptr(depth) if want_depth else None, _ptr(key_hist),
                           1 if deepest_first else 0, _ptr(ws), ws.numel(), _stream()))
    return keys, (depth if want_depth else None), ws


def prev_next_use(keys: torch.Tensor, prev: Optional[torch.Tensor] = None,
                  nxt: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                  key_hist: Optional[torch.Tensor] = None):
    L = lib()
    n = keys.numel()
    dev = _dev()
    if prev is None:
        prev = torch.empty(n, dtype=torch.int32, device=dev)
    if nxt is None:
        nxt = torch.empty(n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(L.pc_prev_next_use_ws(n))
    check(L.pc_prev_next_use(_ptr(keys), n, _ptr(prev), _ptr(nxt), _ptr(key_hist), _ptr(ws), ws.numel(),
                             _stream()))
    return prev, nxt, ws


def high_key_passes_ran(ws: torch.Tensor) -> bool:
    """Whether the last pc_prev_next_use call on this workspace also sorted by
    the high 32 key bits (workspace word 1, decided on the device).
    Synchronises the current stream."""
    torch.cuda.current_stream().synchronize()
    return bool(int(ws[4:8].view(torch.int32).item()))


def prev_next_chained(keys: torch.Tensor, blk_off: torch.Tensor, prev: Optional[torch.Tensor] = None,
                      nxt: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                      key_hist: Optional[torch.Tensor] = None, deepest_first: bool = False,
                      prev_only: bool = False):
    """pc_prev_next_chained: the same prev / next as prev_next_use for keys
    laid out per request as hash_blocks writes them; the path is chosen on
    the device (no synchronisation).  With ``prev_only`` (PC_PREV_ONLY) next
    is scratch and unspecified afterwards."""
    L = lib()
    n = keys.numel()
    n_seqs = blk_off.numel() - 1
    dev = _dev()
    if prev is None:
        prev = torch.empty(n, dtype=torch.int32, device=dev)
    if nxt is None:
        nxt = torch.empty(n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(L.pc_prev_next_chained_ws(n, n_seqs))
    check(L.pc_prev_next_chained(_ptr(keys), n, _ptr(blk_off), n_seqs,
                                 (PREV_ONLY if prev_only else 0) | (DEEPEST_FIRST if deepest_first else 0),
                                 _ptr(prev), _ptr(nxt), _ptr(key_hist), _ptr(ws), ws.numel(), _stream()))
    return prev, nxt, ws


def chained_info(ws: torch.Tensor) -> dict:
    """What the last pc_prev_next_chained call on this workspace did: whether
    the generic prev/next ran over all keys (and why), and how many accesses
    went through the generic prev/next of the unresolved ones.  Synchronises."""
    torch.cuda.current_stream().synchronize()
    w = ws[:32].view(torch.int32).cpu().tolist()
    return {"generic": bool(w[1]), "unresolved": w[2] & 0xFFFFFFFF, "reason": w[3],
            "high_anchor": bool(w[6]), "high_unresolved": bool(w[7])}


def stack_distance(prev: torch.Tensor, nxt: torch.Tensor, dist: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None):
    L = lib()
    n = prev.numel()
    if dist is None:
        dist = torch.empty(n, dtype=torch.int32, device=_dev())
    if ws is None:
        ws = workspace(L.pc_stack_distance_ws(n))
    check(L.pc_stack_distance(_ptr(prev), _ptr(nxt), n, _ptr(dist), _ptr(ws), ws.numel(), _stream()))
    return dist, ws


def stack_distance_noalloc(prev: torch.Tensor, nxt: torch.Tensor, dist: torch.Tensor):
    """pc_stack_distance_noalloc: the same distances as stack_distance into a
    caller-provided ``dist``, with the library's own fixed device scratch
    (nothing is allocated; calls on one GPU must not overlap)."""
    check(lib().pc_stack_distance_noalloc(_ptr(prev), _ptr(nxt), prev.numel(), _ptr(dist), _stream()))
    return dist


def stack_distance_noalloc_max_n() -> int:
    return int(lib().pc_stack_distance_noalloc_max_n())


def stack_distance_runs(prev: torch.Tensor, nxt: torch.Tensor, dist: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None):
    """pc_stack_distance_runs: the same distances as stack_distance, counted
    over the runs of the prev stream, or by the dominance count when there
    are too many runs (chosen on the device; no synchronisation)."""
    L = lib()
    n = prev.numel()
    if dist is None:
        dist = torch.empty(n, dtype=torch.int32, device=_dev())
    if ws is None:
        ws = workspace(L.pc_stack_distance_runs_ws(n))
    check(L.pc_stack_distance_runs(_ptr(prev), _ptr(nxt), n, _ptr(dist), _ptr(ws), ws.numel(), _stream()))
    return dist, ws


def runs_info(ws: torch.Tensor) -> dict:
    """What the last pc_stack_distance_runs call on this workspace did.
    Synchronises."""
    torch.cuda.current_stream().synchronize()
    w = ws[:16].view(torch.int32).cpu().tolist()
    return {"generic": bool(w[1]), "runs": w[2] & 0xFFFFFFFF, "cold": w[3] & 0xFFFFFFFF}


def request_order(keys: torch.Tensor, blk_off: torch.Tensor, depth: Optional[torch.Tensor] = None,
                  keys_out: Optional[torch.Tensor] = None, depth_out: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None):
    """pc_request_order: every request's accesses reversed (deepest block
    first), the recency order of request-level residency."""
    L = lib()
    n = keys.numel()
    n_seqs = blk_off.numel() - 1
    dev = _dev()
    if keys_out is None:
        keys_out = torch.empty(n, dtype=torch.int64, device=dev)
    if depth is not None and depth_out is None:
        depth_out = torch.empty(n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = workspace(L.pc_request_order_ws())
    check(L.pc_request_order(_ptr(keys), _ptr(depth), _ptr(blk_off), n_seqs, n, _ptr(keys_out),
                             _ptr(depth_out) if depth is not None else None, _ptr(ws), ws.numel(),
                             _stream()))
    return keys_out, depth_out, ws


def stack_distance_req(prev: torch.Tensor, dist: torch.Tensor, blk_off: torch.Tensor,
                       dist_req: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """pc_stack_distance_req: request-level stack distances from prev and
    dist of the request-ordered accesses."""
    L = lib()
    n = prev.numel()
    n_seqs = blk_off.numel() - 1
    if dist_req is None:
        dist_req = torch.empty(n, dtype=torch.int32, device=_dev())
    if ws is None:
        ws = workspace(L.pc_stack_distance_req_ws())
    check(L.pc_stack_distance_req(_ptr(prev), _ptr(dist), _ptr(blk_off), n_seqs, n,
                                  _ptr(dist_req), _ptr(ws), ws.numel(), _stream()))
    return dist_req, ws


def stack_distance_session(prev: torch.Tensor, blk_off: torch.Tensor, session: torch.Tensor,
                           dist_sess: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """pc_stack_distance_session: session-level distances from prev (request
    order), the request table and the session of every request."""
    L = lib()
    n = prev.numel()
    n_seqs = blk_off.numel() - 1
    if session.numel() != n_seqs:
        raise PcError("one session id per request expected")
    if dist_sess is None:
        dist_sess = torch.empty(n, dtype=torch.int32, device=_dev())
    if ws is None:
        ws = workspace(L.pc_stack_distance_session_ws(n, n_seqs))
    check(L.pc_stack_distance_session(_ptr(prev), _ptr(blk_off), _ptr(session), n_seqs, n, _ptr(dist_sess),
                                      _ptr(ws), ws.numel(), _stream()))
    return dist_sess, ws


FREQ_CLASSES = 32


def reuse_profile(prev: torch.Tensor, nxt: torch.Tensor, blk_off: torch.Tensor, ts_us: torch.Tensor,
                  edges: torch.Tensor, freq_max: int, out: Optional[dict] = None, ws: Optional[torch.Tensor] = None):
    """pc_reuse_profile: reuse-interval, lifetime, frequency and
    lifetime-by-frequency-class histograms (int64 tensors of uint64)."""
    L = lib()
    n = prev.numel()
    n_seqs = blk_off.numel() - 1
    k = edges.numel()
    dev = _dev()
    if out is None:
        out = {"interval": torch.empty(k + 1, dtype=torch.int64, device=dev),
               "lifetime": torch.empty(k + 1, dtype=torch.int64, device=dev),
               "freq": torch.empty(freq_max + 1, dtype=torch.int64, device=dev),
               "life_by_class": torch.empty(FREQ_CLASSES * (k + 1), dtype=torch.int64, device=dev)}
    if ws is None:
        ws = workspace(L.pc_reuse_profile_ws(n))
    check(L.pc_reuse_profile(_ptr(prev), _ptr(nxt), _ptr(blk_off), _ptr(ts_us), n_seqs, n, _ptr(edges), k,
                             freq_max, _ptr(out["interval"]), _ptr(out["lifetime"]), _ptr(out["freq"]),
                             _ptr(out["life_by_class"]), _ptr(ws), ws.numel(), _stream()))
    return out, ws


def session_profile(blk_off: torch.Tensor, session: torch.Tensor, ts_us: torch.Tensor, n: int,
                    edges: torch.Tensor, fp_max: int, rq_max: int, out: Optional[dict] = None,
                    ws: Optional[torch.Tensor] = None):
    """pc_session_profile: footprint, request-count, duration and gap
    histograms over sessions (int64 tensors of uint64)."""
    L = lib()
    n_seqs = blk_off.numel() - 1
    k = edges.numel()
    dev = _dev()
    if out is None:
        out = {"footprint": torch.empty(fp_max + 1, dtype=torch.int64, device=dev),
               "requests": torch.empty(rq_max + 1, dtype=torch.int64, device=dev),
               "duration": torch.empty(k + 1, dtype=torch.int64, device=dev),
               "gap": torch.empty(k + 1, dtype=torch.int64, device=dev)}
    if ws is None:
        ws = workspace(L.pc_session_profile_ws(n_seqs))
    check(L.pc_session_profile(_ptr(blk_off), _ptr(session), _ptr(ts_us), n_seqs, n, _ptr(edges), k, fp_max,
                               rq_max, _ptr(out["footprint"]), _ptr(out["requests"]), _ptr(out["duration"]),
                               _ptr(out["gap"]), _ptr(ws), ws.numel(), _stream()))
    return out, ws


def hists_to_host(out: dict) -> dict:
    """Device histograms -> lists of python ints."""
    return {name: [int(x) for x in as_u64(t).tolist()] for name, t in out.items()}


def mrc_weighted(dist: torch.Tensor, caps: torch.Tensor, depth: Optional[torch.Tensor] = None,
                 nxt: Optional[torch.Tensor] = None, alpha: int = 1, beta: int = 0,
                 out: Optional[dict] = None, ws: Optional[torch.Tensor] = None):
    """pc_mrc_weighted: per-bin count, depthsum, cost (lo/hi) and next-use
    histogram as int64 tensors of n_caps+1 entries (uint64 bit patterns);
    the next-use histogram is all zero when ``nxt`` is None."""
    L = lib()
    n = dist.numel()
    k = caps.numel()
    dev = _dev()
    if out is None:
        out = {name: torch.empty(k + 1, dtype=torch.int64, device=dev)
               for name in ("count", "depthsum", "cost_lo", "cost_hi", "nextuse")}
    if ws is None:
        ws = workspace(L.pc_mrc_weighted_ws(n, k))
    check(L.pc_mrc_weighted(_ptr(dist), _ptr(depth), _ptr(nxt), n, _ptr(caps), k,
                            alpha & (2 ** 64 - 1), beta & (2 ** 64 - 1), _ptr(out["count"]),
                            _ptr(out["depthsum"]), _ptr(out["cost_lo"]), _ptr(out["cost_hi"]),
                            _ptr(out["nextuse"]), _ptr(ws), ws.numel(),
                            _stream()))
    return out, ws


def mrc_weighted_layout(dist: torch.Tensor, caps: torch.Tensor, blk_off: torch.Tensor,
                        nxt: Optional[torch.Tensor] = None, alpha: int = 1, beta: int = 0,
                        out: Optional[dict] = None, ws: Optional[torch.Tensor] = None, deepest_first: bool = False):
    """pc_mrc_weighted_layout: as mrc_weighted with depth[t] = t - blk_off[r]
    for the request r holding t (the ascending layout of hash_blocks), or
    blk_off[r + 1] - 1 - t with ``deepest_first``."""
    L = lib()
    n = dist.numel()
    k = caps.numel()
    dev = _dev()
    if out is None:
        out = {name: torch.empty(k + 1, dtype=torch.int64, device=dev)
               for name in ("count", "depthsum", "cost_lo", "cost_hi", "nextuse")}
    if ws is None:
        ws = workspace(L.pc_mrc_weighted_layout_ws(n, k))
    check(L.pc_mrc_weighted_layout(_ptr(dist), _ptr(blk_off), blk_off.numel() - 1,
                                   DEEPEST_FIRST if deepest_first else 0, _ptr(nxt), n, _ptr(caps), k,
                                   alpha & (2 ** 64 - 1), beta & (2 ** 64 - 1), _ptr(out["count"]),
                                   _ptr(out["depthsum"]), _ptr(out["cost_lo"]), _ptr(out["cost_hi"]),
                                   _ptr(out["nextuse"]), _ptr(ws), ws.numel(), _stream()))
    return out, ws


def belady(nxt: torch.Tensor, caps: torch.Tensor, depth: Optional[torch.Tensor] = None, flags: bool = False,
           out: Optional[dict] = None, ws: Optional[torch.Tensor] = None):
    """pc_belady: hits and depth sums of Belady's MIN at every capacity
    (int64 tensors of uint64); with ``flags`` also the per-access hit flags
    (uint8 [n_caps, n])."""
    L = lib()
    n = nxt.numel()
    k = caps.numel()
    dev = _dev()
    if out is None:
        out = {"hits": torch.empty(k, dtype=torch.int64, device=dev),
               "depthsum": torch.empty(k, dtype=torch.int64, device=dev)}
    if flags and "flags" not in out:
        out["flags"] = torch.empty((k, n), dtype=torch.uint8, device=dev)
    if ws is None:
        ws = workspace(L.pc_belady_ws(n, k))
    check(L.pc_belady(_ptr(nxt), _ptr(depth), n, _ptr(caps), k, _ptr(out["hits"]), _ptr(out["depthsum"]),
                      _ptr(out.get("flags")) if flags else None, _ptr(ws), ws.numel(), _stream()))
    return out, ws


# ------------------------------------------------------------- paged cache

# PC_BF16, PC_F16, PC_FP8_E4M3, PC_FP4_E2M1
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}
if hasattr(torch, "float4_e2m1fn_x2"):   # newer than the other types: without it there are no caches in 4 bits
    _DTYPES[torch.float4_e2m1fn_x2] = 3
_INTS = (torch.int32, torch.uint32)
_MAX_KV = 0x7FFF0000


def _stream_of(t: torch.Tensor):
    """The current stream of a tensor's device, without the objects around it (a few
    microseconds, as much as a small call's kernels take)."""
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _scratch(nbytes: int, t: torch.Tensor) -> torch.Tensor:
    return t.new_empty((nbytes,), dtype=torch.uint8)


def _table(t: torch.Tensor, what: str, rows: int):
    """A table of 32-bit integers, [rows, columns] with the columns contiguous: (address, row stride)."""
    if not t.is_cuda:
        raise PcError("expected a GPU tensor")
    shape, stride = t.shape, t.stride()
    if t.dtype not in _INTS or len(shape) != 2 or shape[0] != rows or (shape[1] > 1 and stride[1] != 1):
        raise PcError("%s: expected [%d, columns] of 32-bit integers, columns contiguous" % (what, rows))
    return t.data_ptr(), stride[0] if rows > 1 else shape[1]


def _index(t: torch.Tensor, what: str, n: int):
    if t.dtype not in _INTS or t.shape != (n,):
        raise PcError("%s: expected [%d] of 32-bit integers" % (what, n))
    return _ptr(t)


def _rows(t: torch.Tensor, what: str, shape):
    """New tokens [rows, heads, head_dim], head_dim contiguous: (address, row stride, head stride)."""
    if not t.is_cuda:
        raise PcError("expected a GPU tensor")
    stride = t.stride()
    if t.shape != shape or stride[2] != 1:
        raise PcError("%s: expected %s, the last dimension contiguous" % (what, list(shape)))
    return t.data_ptr(), stride[0] if shape[0] > 1 else shape[2], stride[1] if shape[1] > 1 else shape[2]


def _no_gradient():
    """There is no backward pass: what autograd would follow is refused rather than cut off."""
    if torch.is_grad_enabled():
        raise PcError("no backward pass: call under torch.no_grad() or detach what requires a gradient")


def _room(page_table: torch.Tensor, cache, max_kv: Optional[int]) -> int:
    room = page_table.shape[1] * cache.page_size
    if max_kv is None:
        return min(room, _MAX_KV)
    if not 0 <= max_kv <= min(room, _MAX_KV):
        raise PcError("max_kv: the page table has fewer slots, or more than 2^31 - 2^16")
    return max_kv


class PagedCache:
    """A paged cache of KV blocks (``pc_kv_cache``) over two tensors [page, head,
    slot, head_dim] of one type and one set of strides, head_dim contiguous: pages
    kept as [page, slot, head, head_dim] go in as ``x.transpose(1, 2)``.  bfloat16,
    float16, float8_e4m3fn with ``k_scale`` and ``v_scale`` (float32, one per head), or
    float4_e2m1fn_x2 ([page, head, slot, head_dim / 2], two codes an element) with scales
    [page, head, slot, head_dim / 32] of float8_e8m0fnu (or uint8, its bits) whose strides are
    a sixteenth of the codes'; bytes of a plain buffer go in as ``x.view(torch.float4_e2m1fn_x2)``.
    The calls on it have no backward pass and refuse tensors that require a gradient
    (outside of ``torch.no_grad()``)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        dtype, shape, stride = _DTYPES.get(k.dtype), k.shape, k.stride()
        if len(shape) != 4 or v.shape != shape or v.dtype != k.dtype or dtype is None:
            raise PcError("expected two tensors [page, head, slot, head_dim] of bfloat16, float16, float8_e4m3fn or "
                          "float4_e2m1fn_x2")
        if not (k.is_cuda and v.is_cuda):
            raise PcError("expected a GPU tensor")
        if stride[3] != 1 or (v.stride() != stride and any(a != b for a, b, n in zip(stride, v.stride(), shape) if n > 1)):
            raise PcError("expected equal strides of k and v, head_dim contiguous")
        if (k_scale is None) != (dtype < 2) or (v_scale is None) != (dtype < 2):
            raise PcError("k_scale and v_scale go with float8_e4m3fn and float4_e2m1fn_x2")
        if dtype == 3:
            shape = (shape[0], shape[1], shape[2], 2 * shape[3])
            stride = (2 * stride[0], 2 * stride[1], 2 * stride[2], 1)
            self._block_scales(k_scale, shape, stride, v_scale)
        else:
            for x in (k_scale, v_scale):
                if x is not None and (x.dtype != torch.float32 or x.shape != shape[1:2]):
                    raise PcError("expected one float32 scale per head")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._grad = k.requires_grad or v.requires_grad or (
            k_scale is not None and (k_scale.requires_grad or v_scale.requires_grad))
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = shape
        if 1 in shape:   # the stride of a dimension of one is anything
            stride = [s if n > 1 else self.head_dim for s, n in zip(stride, shape)]
        if dtype == 3:
            ka, va = k_scale.data_ptr(), v_scale.data_ptr()
        else:
            ka, va = _ptr(k_scale), _ptr(v_scale)
        self._c = _KvCache(k.data_ptr(), v.data_ptr(), ka, va, stride[0], stride[1], stride[2], dtype, self.n_pages,
                           self.page_size, self.n_kv_heads, self.head_dim)
        self._at = ctypes.addressof(self._c)

    @staticmethod
    def _block_scales(k_scale, shape, stride, v_scale):
        """Those of elements i .. i + 31 lie at i / 32 (pc_kv_cache), so the strides follow from the codes'."""
        pages, heads, slots, dim = shape
        blocks = (pages, heads, slots, dim // 32)
        for x in (k_scale, v_scale):
            if (x.dtype is not torch.uint8 and x.dtype is not torch.float8_e8m0fnu) or x.shape != blocks or not x.is_cuda:
                raise PcError("expected scales %s of float8_e8m0fnu or uint8 on the GPU" % list(blocks))
            a, b, c, d = x.stride()
            if ((32 * a != stride[0] and pages > 1) or (32 * b != stride[1] and heads > 1) or
                    (32 * c != stride[2] and slots > 1) or (d != 1 and dim > 32)):
                raise PcError("scales: expected a sixteenth of the codes' strides")


def kv_append(cache: PagedCache, page_table: torch.Tensor, kv_len: torch.Tensor, q_off: torch.Tensor,
              k: torch.Tensor, v: torch.Tensor, max_kv: Optional[int] = None, ws: Optional[torch.Tensor] = None):
    """pc_kv_append: rows q_off[s] .. q_off[s + 1] - 1 of ``k`` and ``v`` ([rows, head,
    head_dim]) into the last slots of the kv_len[s] of sequence s."""
    L = lib()
    if k.requires_grad or v.requires_grad or cache._grad:
        _no_gradient()
    n_seqs = kv_len.shape[0]
    table, stride = _table(page_table, "page_table", n_seqs)
    max_kv = _room(page_table, cache, max_kv)
    dtype = _DTYPES.get(k.dtype)
    if dtype is None or v.dtype != k.dtype:
        raise PcError("expected k and v of one type, bfloat16 or float16")
    shape = (k.shape[0], cache.n_kv_heads, cache.head_dim)
    ka, kr, kh = _rows(k, "k", shape)
    va, vr, vh = _rows(v, "v", shape)
    if ws is None:
        ws = _scratch(L.pc_kv_append_ws(), k)
    check(L.pc_kv_append(cache._at, table, stride, _index(kv_len, "kv_len", n_seqs), _index(q_off, "q_off", n_seqs + 1),
                         n_seqs, shape[0], max_kv, ka, kr, kh, va, vr, vh, dtype, _ptr(ws), ws.numel(), _stream_of(k)))
    return ws


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     trained: int = 0, slow: float = 1.0, fast: float = 32.0) -> np.ndarray:
    """Angles a position of the rot_dim / 2 pairs of dimensions, float64 on the host:
    f_i = base^(-2 i / rot_dim).  For contexts ``factor`` times longer than trained on, ``scaling``:
    "linear"  f_i / factor (positions interpolated; Chen et al. 2023);
    "base"    the base grown by factor^(rot_dim / (rot_dim - 2)), which divides the last f_i by factor and keeps the first;
    "ramp"    by parts (Peng et al. 2023): a pair that makes t = ``trained`` f_i / (2 pi) turns over the context that was
              trained keeps its f_i where t >= fast, takes f_i / factor where t <= slow, and in between
              (1 - g) f_i / factor + g f_i with g = (t - slow) / (fast - slow).
    A checkpoint whose ramp runs otherwise, such as over i between two bounds rounded to whole numbers, needs
    frequencies of its own: ``rope_table`` takes any array.  The ramp's paper scales queries and keys, too, so that
    their products grow with the context: ``rope_table(magnitude=0.1 * math.log(factor) + 1)``.
    """
    if rot_dim < 2 or rot_dim % 2:
        raise PcError("rot_dim: expected an even number of dimensions")
    if not (math.isfinite(base) and base > 0 and math.isfinite(factor) and factor > 0):
        raise PcError("base and factor: expected numbers above 0")
    if scaling not in (None, "none", "linear", "base", "ramp"):
        raise PcError("scaling: expected none, linear, base or ramp")
    base = np.float64(base)
    with np.errstate(over="ignore", invalid="ignore"):
        if scaling == "base" and rot_dim > 2:
            base = base * np.float64(factor) ** (rot_dim / (rot_dim - 2))
        freq = base ** (np.arange(0, rot_dim, 2) / -float(rot_dim))
        if scaling == "linear":
            freq = freq / factor
        elif scaling == "ramp":
            if not (trained > 0 and fast > slow):
                raise PcError("ramp: expected the trained length, and slow < fast")
            keep = (freq * (trained / (2 * math.pi)) - slow) / (fast - slow)
            keep = np.minimum(np.maximum(keep, 0.0), 1.0)
            freq = freq * (keep + (1 - keep) / factor)
    if not (np.isfinite(base) and np.isfinite(freq).all()):
        raise PcError("base, factor or ramp: the angles are past what 64 bits hold")
    return freq


def rope_table(freq, n_pos: int, first: int = 0, magnitude: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """pc_rope_table: [n_pos, pairs, 2] float32, ``magnitude`` times the cosine and sine of
    the angles (first + p) freq[i].  ``freq`` is a float64 array on the host."""
    L = lib()
    freq = np.ascontiguousarray(freq, dtype=np.float64)
    if freq.ndim != 1 or not 0 <= n_pos < NONE or not 0 <= first < NONE:
        raise PcError("expected one frequency a pair, and positions below 2^32 - 1")
    shape = (n_pos, freq.size, 2)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device="cuda")
    elif out.dtype != torch.float32 or out.shape != shape:
        raise PcError("out: expected %s float32" % list(shape))
    check(L.pc_rope_table(freq.ctypes.data, freq.size, first, n_pos, magnitude, _ptr(out), _stream_of(out)))
    return out


def _rotation(table: torch.Tensor, pos: Optional[torch.Tensor], n_rows: int, flags: int) -> _Rotation:
    if table.dtype != torch.float32 or len(table.shape) != 3 or table.shape[2] != 2 or table.shape[0] >= NONE:
        raise PcError("table: expected [positions, pairs, 2] float32")
    return _Rotation(_ptr(table), None if pos is None else _index(pos, "pos", n_rows), table.shape[0], 2 * table.shape[1], flags)


def rope(x: torch.Tensor, table: torch.Tensor, pos: Optional[torch.Tensor] = None, interleaved: bool = False,
         transpose: bool = False, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """pc_rope: rows ``x`` [rows, head, head_dim] turned by the angles of their positions (``pos``, 32-bit integers;
    their numbers if not given), in the first 2 * pairs dimensions of every head.  ``transpose`` turns back: it
    takes the gradient of the result to that of ``x``.  ``out`` may be ``x``.  Returns (out, ws)."""
    L = lib()
    if x.requires_grad or table.requires_grad:
        _no_gradient()
    dtype, shape = _DTYPES.get(x.dtype), x.shape
    if len(shape) != 3 or dtype is None:
        raise PcError("expected x as [rows, heads, head_dim] of bfloat16 or float16")
    xa, xr, xh = _rows(x, "x", shape)
    if out is None:
        out = x.new_empty(shape)
        oa, o_r, oh = out.data_ptr(), shape[1] * shape[2], shape[2]
    else:
        if out.dtype != x.dtype:
            raise PcError("out: expected x's type")
        oa, o_r, oh = _rows(out, "out", shape)
    turn = _rotation(table, pos, shape[0], (ROPE_INTERLEAVED if interleaved else 0) | (ROPE_TRANSPOSE if transpose else 0))
    if ws is None:
        ws = _scratch(L.pc_rope_ws(), x)
    check(L.pc_rope(ctypes.addressof(turn), xa, xr, xh, oa, o_r, oh, dtype, shape[0], shape[1], shape[2], _ptr(ws), ws.numel(),
                    _stream_of(x)))
    return out, ws


def kv_append_rope(cache: PagedCache, page_table: torch.Tensor, kv_len: torch.Tensor, q_off: torch.Tensor,
                   k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, pos: Optional[torch.Tensor] = None,
                   interleaved: bool = False, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                   max_kv: Optional[int] = None, ws: Optional[torch.Tensor] = None):
    """pc_kv_append_rope: ``kv_append`` of keys turned by the angles of their positions (``pos``, 32-bit integers, one
    per row; their slots if not given), and in the same launch the rows' queries ``q`` [rows, query head, head_dim],
    to ``q_out`` (which may be ``q``).  Returns (q_out or None, ws)."""
    L = lib()
    if k.requires_grad or v.requires_grad or table.requires_grad or cache._grad or (q is not None and q.requires_grad):
        _no_gradient()
    n_seqs = kv_len.shape[0]
    pages, stride = _table(page_table, "page_table", n_seqs)
    max_kv = _room(page_table, cache, max_kv)
    dtype = _DTYPES.get(k.dtype)
    if dtype is None or v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        raise PcError("expected q, k and v of one type, bfloat16 or float16")
    shape = (k.shape[0], cache.n_kv_heads, cache.head_dim)
    ka, kr, kh = _rows(k, "k", shape)
    va, vr, vh = _rows(v, "v", shape)
    qa = qr = qh = oa = o_r = oh = heads = 0
    if q is not None:
        heads = q.shape[1] if len(q.shape) == 3 else 0
        q_shape = (shape[0], heads, shape[2])
        qa, qr, qh = _rows(q, "q", q_shape)
        if q_out is None:
            q_out = q.new_empty(q_shape)
        elif q_out.dtype != q.dtype:
            raise PcError("q_out: expected q's type")
        oa, o_r, oh = _rows(q_out, "q_out", q_shape)
    elif q_out is not None:
        raise PcError("q_out goes with q")
    turn = _rotation(table, pos, shape[0], ROPE_INTERLEAVED if interleaved else 0)
    if ws is None:
        ws = _scratch(L.pc_kv_append_rope_ws(), k)
    check(L.pc_kv_append_rope(cache._at, pages, stride, _index(kv_len, "kv_len", n_seqs), _index(q_off, "q_off", n_seqs + 1),
                              n_seqs, shape[0], max_kv, ctypes.addressof(turn), ka, kr, kh, va, vr, vh, qa or None, qr, qh,
                              oa or None, o_r, oh, heads, dtype, _ptr(ws), ws.numel(), _stream_of(k)))
    return q_out, ws


def attn_paged(q: torch.Tensor, cache: PagedCache, page_table: torch.Tensor, kv_len: torch.Tensor,
               q_off: torch.Tensor, max_q: int, max_kv: Optional[int] = None, scale: Optional[float] = None,
               causal: bool = True, window: int = 0, out: Optional[torch.Tensor] = None, want_lse: bool = False,
               lse: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
               weight_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """pc_attn_paged: attention of the new tokens ``q`` [rows, query head, head_dim]
    over the cache, which holds their keys and values already.  ``max_q`` and
    ``max_kv`` bound a sequence's new rows and its length (max_kv: the page table's
    room if not given); ``scale`` is 1 / sqrt(head_dim) if not given.  Returns
    (out, lse or None, weight_out or None, ws); the accumulated weights
    ([sequence, kv head, max_kv] float32) are formed when ``weight`` or ``weight_out``
    is given."""
    L = lib()
    if q.requires_grad or cache._grad or (weight is not None and weight.requires_grad):
        _no_gradient()
    n_seqs = kv_len.shape[0]
    table, stride = _table(page_table, "page_table", n_seqs)
    max_kv = _room(page_table, cache, max_kv)
    dtype, shape = _DTYPES.get(q.dtype), q.shape
    if not 0 <= window <= NONE or not 0 <= max_q <= NONE:
        raise PcError("window and max_q: expected at least 0 and below 2^32")
    if len(shape) != 3 or dtype is None or shape[2] != cache.head_dim:
        raise PcError("expected q as [rows, heads, %d] of bfloat16 or float16" % cache.head_dim)
    n_rows, n_heads, dim = shape
    qa, qr, qh = _rows(q, "q", shape)
    if out is None:
        out = q.new_empty(shape)
        oa, o_r, oh = out.data_ptr(), n_heads * dim, dim
    else:
        if out.dtype != q.dtype:
            raise PcError("out: expected q's type")
        oa, o_r, oh = _rows(out, "out", shape)
    if lse is None and want_lse:
        lse = q.new_empty((n_rows, n_heads), dtype=torch.float32)
    elif lse is not None and (lse.dtype != torch.float32 or lse.shape != (n_rows, n_heads)):
        raise PcError("lse: expected [rows, heads] float32")
    weight_stride = 0
    if weight is not None or weight_out is not None:
        if weight_out is None:
            weight_out = torch.empty_like(weight)
        weight_stride = weight_out.shape[-1]
        for name, w in (("weight", weight), ("weight_out", weight_out)):
            if w is not None and (w.dtype != torch.float32 or w.shape != (n_seqs, cache.n_kv_heads, weight_stride) or
                                  weight_stride < max_kv):
                raise PcError("%s: expected [sequences, kv heads, at least max_kv] float32" % name)
    if ws is None:
        ws = _scratch(L.pc_attn_paged_ws(n_seqs, n_rows, max_q, max_kv, n_heads, cache.n_kv_heads, dim,
                                         1 if weight_out is not None else 0), q)
    check(L.pc_attn_paged(cache._at, table, stride, _index(kv_len, "kv_len", n_seqs), _index(q_off, "q_off", n_seqs + 1),
                          n_seqs, n_rows, max_q, max_kv, qa, qr, qh, dtype, n_heads,
                          dim ** -0.5 if scale is None else scale, 1 if causal else 0, window, oa, o_r, oh, _ptr(lse),
                          _ptr(weight), _ptr(weight_out), weight_stride, _ptr(ws), ws.numel(), _stream_of(q)))
    return out, lse, weight_out, ws


def kv_evict(cache: PagedCache, page_table: torch.Tensor, kv_len: torch.Tensor, weight: torch.Tensor, budget: int,
             recent: int, dst_table: Optional[torch.Tensor] = None, max_kv: Optional[int] = None,
             out: Optional[dict] = None, ws: Optional[torch.Tensor] = None):
    """pc_kv_evict: per (sequence, head) the last ``recent`` slots and those of the
    largest ``weight`` ([sequence, kv head, at least max_kv] float32), ``budget`` in all, in slot order.
    Their keys and values move to the pages of ``dst_table`` when it is given; slots are
    numbered anew, and a later ``attn_paged(window=...)`` counts kept slots.  Returns
    {"kept" (int32, -1 behind the last), "weight", "new_len", "ws"}."""
    L = lib()
    if weight.requires_grad or cache._grad:
        _no_gradient()
    n_seqs = kv_len.shape[0]
    if not 1 <= budget <= _MAX_KV or not 0 <= recent <= budget:
        raise PcError("expected a budget of 1 to 2^31 - 2^16, and 0 <= recent <= budget")
    table, stride = _table(page_table, "page_table", n_seqs)
    heads = cache.n_kv_heads
    if weight.dtype != torch.float32 or len(weight.shape) != 3 or weight.shape[:2] != (n_seqs, heads):
        raise PcError("weight: expected [sequences, kv heads, slots] float32")
    if max_kv is None:
        max_kv = min(page_table.shape[1] * cache.page_size, weight.shape[2])
    max_kv = _room(page_table, cache, max_kv)
    if max_kv > weight.shape[2]:
        raise PcError("max_kv: the weights have fewer slots")
    dst, dst_stride = None, 0
    if dst_table is not None:
        dst, dst_stride = _table(dst_table, "dst_table", n_seqs)
        if dst_table.shape[1] * cache.page_size < budget:
            raise PcError("dst_table: room for fewer than budget slots")
    shape = (n_seqs, heads, budget)
    if out is None:
        out = {"kept": weight.new_empty(shape, dtype=torch.int32), "weight": weight.new_empty(shape),
               "new_len": kv_len.new_empty((n_seqs,))}
    else:
        kept, w = out.get("kept"), out.get("weight")
        if kept is None or kept.shape != shape or kept.dtype not in _INTS:
            raise PcError("kept: expected [sequences, kv heads, budget] of 32-bit integers")
        if w is not None and (w.shape != shape or w.dtype != torch.float32):
            raise PcError("weight: expected [sequences, kv heads, budget] float32")
    if ws is None:
        ws = _scratch(L.pc_kv_evict_ws(n_seqs, heads, max_kv), weight)
    check(L.pc_kv_evict(cache._at, table, stride, _index(kv_len, "kv_len", n_seqs), n_seqs, max_kv, _ptr(weight),
                        weight.shape[2], budget, recent, dst, dst_stride, _ptr(out["kept"]), _ptr(out.get("weight")),
                        _index(out["new_len"], "new_len", n_seqs), _ptr(ws), ws.numel(), _stream_of(weight)))
    out["ws"] = ws
    return out


def bins_to_host(out: dict) -> dict:
    """Device bins -> python ints (cost as exact 128-bit integers)."""
    c = as_u64(out["count"]).tolist()
    d = as_u64(out["depthsum"]).tolist()
    lo = as_u64(out["cost_lo"]).tolist()
    hi = as_u64(out["cost_hi"]).tolist()
    nu = as_u64(out["nextuse"]).tolist()
    return {"count": [int(x) for x in c], "depthsum": [int(x) for x in d],
            "cost": [int(h) << 64 | int(l) for l, h in zip(lo, hi)], "nextuse": [int(x) for x in nu]}


def curves(count, cost):
    """Hit ratio and compute-savings ratio at each capacity edge from exact
    integer bins: hits(c_k) = sum count[0..k], saved(c_k) = sum cost[0..k];
    each ratio is one float64 division of exactly rounded integers."""
    n = sum(count)
    total = sum(cost)
    hr, csr = [], []
    h = s = 0
    for k in range(len(count) - 1):
        h += count[k]
        s += cost[k]
        hr.append(float(h) / float(n) if n else 0.0)
        csr.append(float(s) / float(total) if total else 0.0)
    return hr, csr


# --------------------------------------------------------------- profiling

def prof_enable(on: bool = True) -> None:
    lib().pc_prof_enable(1 if on else 0)


def prof_read() -> dict:
    """{kernel: (launches, total_ms)} since the last read (caller syncs)."""
    L = lib()
    n = L.pc_prof_kernel_count()
    la = (ctypes.c_uint64 * n)()
    ms = (ctypes.c_double * n)()
    check(L.pc_prof_read(la, ms, n))
    return {L.pc_prof_kernel_name(i).decode(): (int(la[i]), float(ms[i])) for i in range(n)}


# ---------------------------------------------------------------- pipeline

class Pipeline:
    """All four stages over one trace with buffers and workspaces allocated
    once; ``run()`` enqueues hash -> prev/next -> stack distance -> bins.

    ``residency="access"`` bins the per-access LRU stack distance.
    ``residency="session"`` (whole sessions evicted at once, Sec. 5.3) bins
    the session-level distance instead; it needs ``session``, the session of
    every request, and takes no next-use histogram.
    ``residency="request"`` (every block of a request resident at once,
    Sec. 3.1) hashes each request's blocks straight into recency order
    (deepest block first; ``keys_r`` and ``depth_r`` alias ``keys`` and
    ``depth``), runs prev/next and the stack distance on that order, turns
    the result into the request-level distance and bins that, with depth in
    the same order; the next-use histogram is not taken in that mode.  Its
    bins are valid at capacities of at least the largest request.
    ``with_belady`` (per-access mode) also runs Belady's MIN at every
    capacity on the step's next-use index (``belady_out``).

    The bins take each block's depth from the request layout
    (``mrc_weighted_layout``) and the hash writes no depth (``depth`` and
    ``depth_r`` are None); ``depth_array=True``, and Belady's MIN, keep the
    depth array."""

    def __init__(self, tokens, tok_start, tok_len, blk_off, n_blocks: int, caps,
                 block_size: int = 16, alpha: int = 1, beta: int = 0, with_nextuse: bool = True,
                 residency: str = "access", session: Optional[torch.Tensor] = None, chained: bool = True,
                 with_belady: bool = False, depth_array: bool = False):
        if residency not in ("access", "request", "session"):
            raise PcError("residency must be 'access', 'request' or 'session'")
        if residency == "session" and session is None:
            raise PcError("session-level residency needs the session of every request")
        L = lib()
        dev = _dev()
        self.tokens, self.tok_start, self.tok_len, self.blk_off = tokens, tok_start, tok_len, blk_off
        self.n = int(n_blocks)
        self.B = block_size
        self.caps = caps
        self.alpha, self.beta = alpha, beta
        self.residency = residency
        self.request = residency == "request"
        self.session = session
        self.with_nextuse = with_nextuse and residency == "access"
        self.with_belady = with_belady and residency == "access"
        self.layout_depth = not (depth_array or self.with_belady)
        n = self.n
        self.keys = torch.empty(n, dtype=torch.int64, device=dev)
        self.key_hist = torch.empty(4 * 256, dtype=torch.int32, device=dev)
        self.depth = None if self.layout_depth else torch.empty(n, dtype=torch.int32, device=dev)
        self.prev = torch.empty(n, dtype=torch.int32, device=dev)
        self.next = torch.empty(n, dtype=torch.int32, device=dev)
        self.dist = torch.empty(n, dtype=torch.int32, device=dev)
        k = caps.numel()
        self.bins = {name: torch.empty(k + 1, dtype=torch.int64, device=dev)
                     for name in ("count", "depthsum", "cost_lo", "cost_hi", "nextuse")}
        self.ws_hash = workspace(L.pc_hash_blocks_ws(tok_len.numel()))
        self.chained = chained
        self.ws_pn = workspace(L.pc_prev_next_chained_ws(n, tok_len.numel()) if chained
                               else L.pc_prev_next_use_ws(n))
        if residency == "session":
            self.ws_sd = workspace(L.pc_stack_distance_session_ws(n, tok_len.numel()))
        else:
            self.ws_sd = workspace(L.pc_stack_distance_runs_ws(n) if chained else L.pc_stack_distance_ws(n))
        if self.request:
            self.keys_r, self.depth_r = self.keys, self.depth   # hashed in recency order
            self.dist_req = torch.empty(n, dtype=torch.int32, device=dev)
            self.ws_req = workspace(L.pc_stack_distance_req_ws())
        self.ws_mrc = workspace(L.pc_mrc_weighted_layout_ws(n, k) if self.layout_depth
                                else L.pc_mrc_weighted_ws(n, k))
        if self.with_belady:
            self.belady_out = {"hits": torch.empty(k, dtype=torch.int64, device=dev),
                               "depthsum": torch.empty(k, dtype=torch.int64, device=dev)}
            self.ws_bel = workspace(L.pc_belady_ws(n, k))

    def run(self):
        hash_blocks(self.tokens, self.tok_start, self.tok_len, self.blk_off, self.n, self.B,
                    want_depth=not self.layout_depth, keys=self.keys, depth=self.depth, ws=self.ws_hash,
                    key_hist=self.key_hist, deepest_first=self.request)
        if self.residency == "session":
            self._prev_next(self.keys)
            stack_distance_session(self.prev, self.blk_off, self.session, dist_sess=self.dist, ws=self.ws_sd)
            self._bins(None)
            return
        if not self.request:
            self._prev_next(self.keys)
            self._stack_distance()
            self._bins(self.next if self.with_nextuse else None)
            if self.with_belady:
                belady(self.next, self.caps, self.depth, out=self.belady_out, ws=self.ws_bel)
            return
        self._prev_next(self.keys_r)
        self._stack_distance()
        stack_distance_req(self.prev, self.dist, self.blk_off, dist_req=self.dist_req, ws=self.ws_req)
        if self.layout_depth:
            mrc_weighted_layout(self.dist_req, self.caps, self.blk_off, None, self.alpha, self.beta, out=self.bins,
                                ws=self.ws_mrc, deepest_first=True)
        else:
            mrc_weighted(self.dist_req, self.caps, self.depth_r, None, self.alpha, self.beta,
                         out=self.bins, ws=self.ws_mrc)

    def _bins(self, nxt):
        if self.layout_depth:
            mrc_weighted_layout(self.dist, self.caps, self.blk_off, nxt, self.alpha, self.beta, out=self.bins,
                                ws=self.ws_mrc)
        else:
            mrc_weighted(self.dist, self.caps, self.depth, nxt, self.alpha, self.beta, out=self.bins, ws=self.ws_mrc)

    def _prev_next(self, keys):
        if self.chained:
            # session-level eviction reads no next use
            prev_next_chained(keys, self.blk_off, self.prev, self.next, ws=self.ws_pn, key_hist=self.key_hist,
                              deepest_first=self.request, prev_only=self.residency == "session")
        else:
            prev_next_use(keys, self.prev, self.next, ws=self.ws_pn, key_hist=self.key_hist)

    def _stack_distance(self):
        if self.chained:
            stack_distance_runs(self.prev, self.next, self.dist, ws=self.ws_sd)
        else:
            stack_distance(self.prev, self.next, self.dist, ws=self.ws_sd)

    def high_key_passes_ran(self) -> bool:
        """Whether the last generic prev/next call also sorted by the high 32
        key bits (decided on the device; see pc_prev_next_use).  Synchronises."""
        return high_key_passes_ran(self.ws_pn)

    def chained_info(self) -> dict:
        """What the last chained prev/next did (see chained_info)."""
        return chained_info(self.ws_pn)

    def status(self) -> dict:
        stages = [("hash", self.ws_hash), ("prev_next", self.ws_pn), ("stack_distance", self.ws_sd),
                  ("mrc", self.ws_mrc)]
        if self.request:
            stages.append(("stack_distance_req", self.ws_req))
        if self.with_belady:
            stages.append(("belady", self.ws_bel))
        return {name: workspace_status(ws) for name, ws in stages}


class Profiler:
    """Workload characterisation over one trace (Sec. 4): hash -> prev/next
    -> reuse profile (intervals, lifetimes, frequencies) and session profile
    (footprints, requests, durations, gaps), buffers allocated once."""

    def __init__(self, tokens, tok_start, tok_len, blk_off, n_blocks: int, session, ts_us, edges,
                 block_size: int = 16, freq_max: int = 2048, fp_max: int = 1 << 16, rq_max: int = 2048,
                 chained: bool = True):
        L = lib()
        dev = _dev()
        self.tokens, self.tok_start, self.tok_len, self.blk_off = tokens, tok_start, tok_len, blk_off
        self.session, self.ts_us, self.edges = session, ts_us, edges
        self.n = int(n_blocks)
        self.B = block_size
        self.freq_max, self.fp_max, self.rq_max = freq_max, fp_max, rq_max
        n = self.n
        self.keys = torch.empty(n, dtype=torch.int64, device=dev)
        self.key_hist = torch.empty(4 * 256, dtype=torch.int32, device=dev)
        self.prev = torch.empty(n, dtype=torch.int32, device=dev)
        self.next = torch.empty(n, dtype=torch.int32, device=dev)
        self.ws_hash = workspace(L.pc_hash_blocks_ws(tok_len.numel()))
        self.chained = chained
        self.ws_pn = workspace(L.pc_prev_next_chained_ws(n, tok_len.numel()) if chained
                               else L.pc_prev_next_use_ws(n))
        self.ws_rp = workspace(L.pc_reuse_profile_ws(n))
        self.ws_sp = workspace(L.pc_session_profile_ws(tok_len.numel()))
        k = edges.numel()
        self.reuse = {"interval": torch.empty(k + 1, dtype=torch.int64, device=dev),
                      "lifetime": torch.empty(k + 1, dtype=torch.int64, device=dev),
                      "freq": torch.empty(freq_max + 1, dtype=torch.int64, device=dev),
                      "life_by_class": torch.empty(FREQ_CLASSES * (k + 1), dtype=torch.int64, device=dev)}
        self.sessions = {"footprint": torch.empty(fp_max + 1, dtype=torch.int64, device=dev),
                         "requests": torch.empty(rq_max + 1, dtype=torch.int64, device=dev),
                         "duration": torch.empty(k + 1, dtype=torch.int64, device=dev),
                         "gap": torch.empty(k + 1, dtype=torch.int64, device=dev)}

    def run(self):
        hash_blocks(self.tokens, self.tok_start, self.tok_len, self.blk_off, self.n, self.B,
                    want_depth=False, keys=self.keys, ws=self.ws_hash, key_hist=self.key_hist)
        if self.chained:
            prev_next_chained(self.keys, self.blk_off, self.prev, self.next, ws=self.ws_pn, key_hist=self.key_hist)
        else:
            prev_next_use(self.keys, self.prev, self.next, ws=self.ws_pn, key_hist=self.key_hist)
        reuse_profile(self.prev, self.next, self.blk_off, self.ts_us, self.edges, self.freq_max,
                      out=self.reuse, ws=self.ws_rp)
        session_profile(self.blk_off, self.session, self.ts_us, self.n, self.edges, self.fp_max, self.rq_max,
                        out=self.sessions, ws=self.ws_sp)

    def status(self) -> dict:
        return {name: workspace_status(ws) for name, ws in
                (("hash", self.ws_hash), ("prev_next", self.ws_pn), ("reuse_profile", self.ws_rp),
                 ("session_profile", self.ws_sp))}


def upload_trace(trace, block_size: Optional[int] = None):
    """Copy a pcgen.Trace's arrays to the GPU (input preparation, untimed)."""
    B = block_size or trace.block_size
    off = trace.blk_off(B)
    dev = _dev()
    return dict(tokens=torch.from_numpy(trace.tokens).to(dev),
                tok_start=to_dev_u64(trace.tok_start), tok_len=to_dev_u32(trace.tok_len),
                blk_off=to_dev_u64(off), n_blocks=int(off[-1]), block_size=B,
                session=to_dev_u32(trace.session.astype(np.uint32)),
                ts_us=to_dev_u64(trace.ts_us.astype(np.uint64)))
