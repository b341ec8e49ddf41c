"""ctypes binding of libspecblock.so -- argument marshalling only.

Every function here has the name of the C entry point it calls (include/specblock.h) and does
nothing but turn torch CUDA tensors into device pointers, size the workspace and raise on a
non-zero return code.  All computation happens in the CUDA library; there is no CPU fallback:
if the library is missing or no CUDA device is present these calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

from . import build as _build

SB_MAX_NODES = 128
SB_MAX_DEPTH = 32
SB_KMAX = 16
SB_BF16, SB_F32 = 0, 1

STATUS_NAMES = {0: "SB_OK", 1: "SB_ERR_INVALID_ARG", 2: "SB_ERR_UNSUPPORTED", 3: "SB_ERR_WORKSPACE",
                4: "SB_ERR_INVALID_TREE", 5: "SB_ERR_BOUNDS", 6: "SB_ERR_CUDA", 7: "SB_ERR_NO_PAGES"}


class SbError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)}")


class _TreeBatch(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
        ("page_size", C.c_int32), ("max_pages", C.c_int32), ("kv_capacity", C.c_int64),
        ("num_pages", C.c_int32), ("total_nodes", C.c_int32), ("page_table", C.c_void_p),
        ("prefix_len", C.c_void_p), ("node_offsets", C.c_void_p), ("parent", C.c_void_p),
        ("max_nodes", C.c_int32), ("max_kv_len", C.c_int32),
        ("index_arrays_settled", C.c_int32), ("prefix_rows_settled", C.c_int32),
    ]


_lib = None


def lib_path() -> str:
    return _build.LIB


def _open(path: str):
    lib = C.CDLL(path)
    lib.sb_status_string.restype = C.c_char_p
    lib.sb_version.restype = C.c_int32
    lib.sb_kernel_launch_count.restype = C.c_int64
    for name in ("sb_tree_attention_workspace_bytes", "sb_tree_expand_workspace_bytes",
                 "sb_verify_accept_workspace_bytes", "sb_rank_features_workspace_bytes",
                 "sb_verify_sample_workspace_bytes", "sb_shift_project_workspace_bytes",
                 "sb_fuse_project_workspace_bytes"):
        getattr(lib, name).restype = C.c_size_t
    for name in ("sb_tree_ancestors", "sb_tree_attention", "sb_tree_expand", "sb_verify_accept",
                 "sb_verify_accept_static", "sb_kv_compact", "sb_path_rows", "sb_rank_features", "sb_verifier_signal",
                 "sb_verify_sample", "sb_shift_project", "sb_fuse_project", "sb_tree_expand_features"):
        getattr(lib, name).restype = C.c_int
    # the calls over 8-bit caches and pages take plain integers for pointers (declared argument types)
    P, I, L, Z, F = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    for name, res, args in (
            ("sb_tree_attention_quant", C.c_int, (P, I, P, P, P, L, P, P, I, P, L, P, P, F, I, I, I, P, Z, P, P)),
            ("sb_tree_attention_quant_workspace_bytes", Z, (P, P, I, I, I, I)),
            ("sb_kv_append_quant", C.c_int, (P, P, P, L, L, P, I, P, P, I, I, P, P, P, P)),
            ("sb_pages_workspace_bytes", Z, (P, I)),
            ("sb_pages_fork", C.c_int, (P, I, P, P, P, P, Z, P, P)),
            ("sb_pages_reserve", C.c_int, (P, I, P, P, P, P, P, P, P, Z, P, P)),
            ("sb_pages_release", C.c_int, (P, I, P, P, P, Z, P, P)),
            ("sb_pages_compact", C.c_int, (P, P, P, I, P, P, P, Z, P, P)),
            ("sb_pages_copy", C.c_int, (P, I, I, I, P, P, P, I, P))):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


def load(build_if_missing: bool = True):
    """Load libspecblock.so (building it in-tree with nvcc when it is absent or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build() if build_if_missing else _build.LIB
    if not os.path.exists(path):
        raise RuntimeError("libspecblock.so is not built: run python -m paper_2605_07243_b200.build")
    _lib = _open(path)
    return _lib


_variants = {}


@contextlib.contextmanager
def build_variant(name: str):
    """Inside the block every call of this module goes to another build of the same sources:
    "test" (libspecblock_test.so: the mma.sync and one-warp-per-row attention kernels as independent
    cross-checks, the environment switches SB_ATTN_IMPL / SB_ATTN_TWO_TILES / SB_ATTN_MAX_CLUSTER /
    SB_NO_PDL / SB_DEBUG, and the wait-expiry kernel) or "checked" (libspecblock_checked.so: every
    computed index verified before use).  For tests; the library proper is what load() returns."""
    global _lib
    load()
    if name not in _variants:
        _variants[name] = _open(_build.build(variant=name))
    saved, _lib = _lib, _variants[name]
    try:
        yield _lib
    finally:
        _lib = saved


EXPORTED = ("sb_tree_ancestors", "sb_tree_attention", "sb_tree_attention_workspace_bytes",
            "sb_tree_expand", "sb_tree_expand_workspace_bytes", "sb_verify_accept",
            "sb_verify_accept_workspace_bytes", "sb_verify_accept_static", "sb_kv_compact", "sb_path_rows",
            "sb_rank_features", "sb_rank_features_workspace_bytes", "sb_verifier_signal", "sb_verify_sample",
            "sb_verify_sample_workspace_bytes", "sb_shift_project", "sb_shift_project_workspace_bytes",
            "sb_fuse_project", "sb_fuse_project_workspace_bytes", "sb_tree_expand_features", "sb_status_string",
            "sb_version",
            "sb_kernel_launch_count", "sb_tree_attention_quant", "sb_tree_attention_quant_workspace_bytes",
            "sb_kv_append_quant", "sb_pages_workspace_bytes", "sb_pages_fork", "sb_pages_reserve", "sb_pages_release",
            "sb_pages_compact", "sb_pages_copy")


def _ptr(t: Optional[torch.Tensor], dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code, where):
    if code != 0:
        raise SbError(code, where)


def sb_kernel_launch_count() -> int:
    return int(load().sb_kernel_launch_count())


def sb_version() -> int:
    return int(load().sb_version())


def sb_status_string(code: int) -> str:
    return load().sb_status_string(C.c_int(code)).decode()


@dataclass
class TreeBatch:
    """Device-side description of a ragged batch of trees over one layer's KV cache; mirrors the
    C struct sb_tree_batch field for field.  k_cache / v_cache: bf16 tensors."""
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    k_cache: torch.Tensor
    v_cache: torch.Tensor
    prefix_len: torch.Tensor          # int32 [B]
    node_offsets: torch.Tensor        # int32 [B+1]
    parent: torch.Tensor              # int32 [total_nodes]
    total_nodes: int
    max_nodes: int
    max_kv_len: int
    page_size: int = 0
    kv_capacity: int = 0
    page_table: Optional[torch.Tensor] = None   # int32 [B, max_pages]
    num_pages: int = 0
    max_pages: int = 0

    def c_struct(self, k_cache=None, v_cache=None, settled=False, prefix_settled=False) -> _TreeBatch:
        k = self.k_cache if k_cache is None else k_cache
        v = self.v_cache if v_cache is None else v_cache
        s = _TreeBatch()
        s.batch = self.prefix_len.numel()
        s.n_q_heads, s.n_kv_heads, s.head_dim = self.n_q_heads, self.n_kv_heads, self.head_dim
        s.k_cache = _ptr(k, torch.bfloat16).value
        s.v_cache = _ptr(v, torch.bfloat16).value
        s.page_size, s.max_pages, s.kv_capacity = self.page_size, self.max_pages, self.kv_capacity
        s.num_pages, s.total_nodes = self.num_pages, self.total_nodes
        s.page_table = None if self.page_table is None else _ptr(self.page_table, torch.int32).value
        s.prefix_len = _ptr(self.prefix_len, torch.int32).value
        s.node_offsets = _ptr(self.node_offsets, torch.int32).value
        s.parent = _ptr(self.parent, torch.int32).value
        s.max_nodes, s.max_kv_len = self.max_nodes, self.max_kv_len
        s.index_arrays_settled = 1 if settled else 0
        s.prefix_rows_settled = 1 if (settled and prefix_settled) else 0
        return s


def sb_tree_ancestors(node_offsets, parent, max_nodes, anc_mask=None, depth=None, status=None):
    """-> (anc_mask int32 [total,4] holding the uint32 words, depth int32 [total], status [B])."""
    batch = node_offsets.numel() - 1
    total = parent.numel()
    dev = parent.device
    anc_mask = torch.empty((total, 4), dtype=torch.int32, device=dev) if anc_mask is None else anc_mask
    depth = torch.empty(total, dtype=torch.int32, device=dev) if depth is None else depth
    status = torch.empty(batch, dtype=torch.int32, device=dev) if status is None else status
    rc = load().sb_tree_ancestors(C.c_int32(batch), _ptr(node_offsets, torch.int32),
                                  _ptr(parent, torch.int32), C.c_int32(max_nodes), _ptr(anc_mask),
                                  _ptr(depth, torch.int32), _ptr(status, torch.int32), _stream())
    _check(rc, "sb_tree_ancestors")
    return anc_mask, depth, status


def sb_tree_attention_workspace_bytes(tb: TreeBatch, total_q: int, num_splits: int = 0) -> int:
    s = tb.c_struct()
    return int(load().sb_tree_attention_workspace_bytes(C.byref(s), C.c_int32(total_q),
                                                        C.c_int32(num_splits)))


def sb_tree_attention(tb: TreeBatch, q, out=None, lse=None, *, q_node_begin=None, q_offsets=None,
                      scale=0.0, num_splits=0, workspace=None, status=None, want_lse=True,
                      k_cache=None, v_cache=None, index_arrays_settled=False, prefix_rows_settled=False):
    """q bf16 [total_q, Hq, D] -> (out bf16 like q, lse fp32 [total_q, Hq] or None, status [B]).
    k_cache / v_cache override the batch's layer (same layout) without rebuilding it.
    index_arrays_settled: the kernel enqueued just before this call does not write the batch's index
    arrays (e.g. it is the previous layer's attention): the lengths may be fetched under its tail.
    prefix_rows_settled (with index_arrays_settled): nor does it write cache rows below prefix_len: key
    blocks inside the prefix may be requested under its tail too."""
    total_q = q.shape[0]
    dev = q.device
    out = torch.empty_like(q) if out is None else out
    if lse is None and want_lse:
        lse = torch.empty((total_q, tb.n_q_heads), dtype=torch.float32, device=dev)
    status = torch.empty(tb.prefix_len.numel(), dtype=torch.int32, device=dev) if status is None else status
    s = tb.c_struct(k_cache, v_cache, index_arrays_settled, prefix_rows_settled)
    lib = load()
    if workspace is None:
        need = int(lib.sb_tree_attention_workspace_bytes(C.byref(s), C.c_int32(total_q),
                                                         C.c_int32(num_splits)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    rc = lib.sb_tree_attention(C.byref(s), _ptr(q_node_begin, torch.int32), _ptr(q_offsets, torch.int32),
                               C.c_int32(total_q), _ptr(q, torch.bfloat16), _ptr(out, torch.bfloat16),
                               _ptr(lse, torch.float32), C.c_float(scale), C.c_int32(num_splits),
                               _ptr(workspace), C.c_size_t(workspace.numel() * workspace.element_size()),
                               _ptr(status, torch.int32), _stream())
    _check(rc, "sb_tree_attention")
    return out, lse, status


def sb_verify_accept_workspace_bytes(total_nodes: int, vocab: int) -> int:
    return int(load().sb_verify_accept_workspace_bytes(C.c_int32(total_nodes), C.c_int32(vocab)))


def sb_verify_accept(logits, node_offsets, parent, tok, max_depth, *, vocab=None, workspace=None,
                     out=None):
    """logits [total_nodes, stride] bf16 or fp32 -> dict(amax, accept_len, path_nodes, out_tokens,
    bonus, status) of int32 device tensors (`out` may pass preallocated ones)."""
    total, stride = logits.shape
    vocab = stride if vocab is None else vocab
    batch = node_offsets.numel() - 1
    dev = logits.device
    dt = {torch.bfloat16: SB_BF16, torch.float32: SB_F32}[logits.dtype]
    if out is None:
        i32 = dict(dtype=torch.int32, device=dev)
        out = dict(amax=torch.empty(total, **i32), accept_len=torch.empty(batch, **i32),
                   path_nodes=torch.empty((batch, max_depth + 1), **i32),
                   out_tokens=torch.empty((batch, max_depth + 1), **i32),
                   bonus=torch.empty(batch, **i32), status=torch.empty(batch, **i32))
    lib = load()
    if workspace is None:
        need = sb_verify_accept_workspace_bytes(total, vocab)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    rc = lib.sb_verify_accept(_ptr(logits), C.c_int(dt), C.c_int64(stride), C.c_int32(vocab),
                              C.c_int32(batch), C.c_int32(total), _ptr(node_offsets, torch.int32),
                              _ptr(parent, torch.int32), _ptr(tok, torch.int32), C.c_int32(max_depth),
                              _ptr(out["amax"]), _ptr(out["accept_len"]), _ptr(out["path_nodes"]),
                              _ptr(out["out_tokens"]), _ptr(out["bonus"]), _ptr(workspace),
                              C.c_size_t(workspace.numel()), _ptr(out["status"]), _stream())
    _check(rc, "sb_verify_accept")
    return out


def sb_rank_features_workspace_bytes(n_rows: int, vocab: int) -> int:
    return int(load().sb_rank_features_workspace_bytes(C.c_int32(n_rows), C.c_int32(vocab)))


def sb_rank_features(scores, *, vocab=None, features=None, workspace=None):
    """scores fp32 [R, stride] -> features fp32 [R, 15] (top-10 log-probs, 3 logit gaps, top
    probability, entropy)."""
    n_rows, stride = scores.shape
    vocab = stride if vocab is None else vocab
    dev = scores.device
    features = torch.empty((n_rows, 15), dtype=torch.float32, device=dev) if features is None else features
    if workspace is None:
        workspace = torch.empty(max(sb_rank_features_workspace_bytes(n_rows, vocab), 256), dtype=torch.uint8, device=dev)
    rc = load().sb_rank_features(_ptr(scores, torch.float32), C.c_int64(stride), C.c_int32(n_rows), C.c_int32(vocab),
                                 _ptr(features, torch.float32), _ptr(workspace), C.c_size_t(workspace.numel()),
                                 _stream())
    _check(rc, "sb_rank_features")
    return features


def sb_verifier_signal(scores, node_offsets, child_row, path_nodes, accept_len, bonus, max_depth, signal, *,
                       vocab=None, r_prob=None, status=None):
    """One iteration's term of s = sum (1 - r): signal fp32 [B] is updated in place.
    -> dict(r_prob, signal, status)."""
    n_rows, stride = scores.shape
    vocab = stride if vocab is None else vocab
    batch = node_offsets.numel() - 1
    dev = scores.device
    r_prob = torch.empty(batch, dtype=torch.float32, device=dev) if r_prob is None else r_prob
    status = torch.empty(batch, dtype=torch.int32, device=dev) if status is None else status
    rc = load().sb_verifier_signal(
        _ptr(scores, torch.float32), C.c_int64(stride), C.c_int32(n_rows), C.c_int32(vocab), C.c_int32(batch),
        C.c_int32(child_row.numel()), _ptr(node_offsets, torch.int32), _ptr(child_row, torch.int32),
        _ptr(path_nodes, torch.int32), _ptr(accept_len, torch.int32), _ptr(bonus, torch.int32),
        C.c_int32(max_depth), _ptr(r_prob, torch.float32), _ptr(signal, torch.float32), _ptr(status, torch.int32),
        _stream())
    _check(rc, "sb_verifier_signal")
    return dict(r_prob=r_prob, signal=signal, status=status)


def sb_verify_sample_workspace_bytes(batch: int, vocab: int, total_nodes: int, n_rows: int) -> int:
    return int(load().sb_verify_sample_workspace_bytes(C.c_int32(batch), C.c_int32(vocab), C.c_int32(total_nodes),
                                                       C.c_int32(n_rows)))


def sb_verify_sample(logits, scores, node_offsets, parent, tok, child_row, temperature, u_accept, u_bonus, max_depth,
                     *, vocab=None, workspace=None, out=None):
    """Stochastic tree verification (temperature > 0); the uniforms are inputs.
    -> dict(accept_len, path_nodes, out_tokens, bonus, status)."""
    total, stride = logits.shape
    n_rows, sstride = scores.shape
    vocab = stride if vocab is None else vocab
    batch = node_offsets.numel() - 1
    dev = logits.device
    dt = {torch.bfloat16: SB_BF16, torch.float32: SB_F32}[logits.dtype]
    if out is None:
        i32 = dict(dtype=torch.int32, device=dev)
        out = dict(accept_len=torch.empty(batch, **i32), path_nodes=torch.empty((batch, max_depth + 1), **i32),
                   out_tokens=torch.empty((batch, max_depth + 1), **i32), bonus=torch.empty(batch, **i32),
                   status=torch.empty(batch, **i32))
    if workspace is None:
        workspace = torch.empty(max(sb_verify_sample_workspace_bytes(batch, vocab, total, n_rows), 256), dtype=torch.uint8,
                                device=dev)
    rc = load().sb_verify_sample(
        _ptr(logits), C.c_int(dt), C.c_int64(stride), C.c_int32(vocab), _ptr(scores, torch.float32), C.c_int64(sstride),
        C.c_int32(n_rows), C.c_int32(batch), C.c_int32(total), _ptr(node_offsets, torch.int32),
        _ptr(parent, torch.int32), _ptr(tok, torch.int32), _ptr(child_row, torch.int32), C.c_float(temperature),
        _ptr(u_accept, torch.float32), _ptr(u_bonus, torch.float32), C.c_int32(max_depth), _ptr(out["accept_len"]),
        _ptr(out["path_nodes"]), _ptr(out["out_tokens"]), _ptr(out["bonus"]), _ptr(workspace),
        C.c_size_t(workspace.numel()), _ptr(out["status"]), _stream())
    _check(rc, "sb_verify_sample")
    return out


def sb_shift_project_workspace_bytes(n_rows: int, d: int, d_out: int, block_k: int) -> int:
    return int(load().sb_shift_project_workspace_bytes(C.c_int32(n_rows), C.c_int32(d), C.c_int32(d_out),
                                                       C.c_int32(block_k)))


def sb_shift_project(h, w, block_k, *, out=None, workspace=None, status=None):
    """h bf16 [R, d], w bf16 [d_out, 2d] (block_k > 0) or [d_out, d] (block_k = 0) -> out bf16 [R, d_out]."""
    n_rows, d = h.shape
    d_out = w.shape[0]
    dev = h.device
    out = torch.empty((n_rows, d_out), dtype=torch.bfloat16, device=dev) if out is None else out
    status = torch.zeros(1, dtype=torch.int32, device=dev) if status is None else status
    if w.shape[1] != (2 * d if block_k > 0 else d):
        raise ValueError("w must be [d_out, 2d] with block_k > 0 and [d_out, d] with block_k = 0")
    if workspace is None:
        workspace = torch.zeros(max(sb_shift_project_workspace_bytes(n_rows, d, d_out, block_k), 256), dtype=torch.uint8,
                                device=dev)
    rc = load().sb_shift_project(_ptr(h, torch.bfloat16), _ptr(w, torch.bfloat16), C.c_int32(n_rows), C.c_int32(d),
                                 C.c_int32(d_out), C.c_int32(block_k), _ptr(out, torch.bfloat16), _ptr(workspace),
                                 C.c_size_t(workspace.numel()), _ptr(status, torch.int32), _stream())
    _check(rc, "sb_shift_project")
    return out, status


def sb_fuse_project_workspace_bytes(n_starts: int, block_k: int, d: int, d_out: int, q_term_valid: bool) -> int:
    return int(load().sb_fuse_project_workspace_bytes(C.c_int32(n_starts), C.c_int32(block_k), C.c_int32(d),
                                                      C.c_int32(d_out), C.c_int32(1 if q_term_valid else 0)))


def sb_fuse_project(c, e, q, w, *, gain_c=None, gain_e=None, gain_q=None, eps=1e-6, q_term=None, q_term_valid=False,
                    out=None, workspace=None, status=None):
    """c, e bf16 [S, d], q bf16 [K, d], w bf16 [d_out, 3d] -> out bf16 [S*K, d_out] (row s*K + k).
    q_term fp32 [K, d_out]: written when q_term_valid is false, read (and a third of w skipped) when true."""
    n_starts, d = c.shape
    block_k = q.shape[0]
    d_out = w.shape[0]
    dev = c.device
    if e.shape != c.shape or q.shape[1] != d or w.shape[1] != 3 * d:
        raise ValueError("expected c, e [S, d], q [K, d], w [d_out, 3d]")
    if q_term is not None and tuple(q_term.shape) != (block_k, d_out):
        raise ValueError("q_term must be [K, d_out]")
    out = torch.empty((n_starts * block_k, d_out), dtype=torch.bfloat16, device=dev) if out is None else out
    status = torch.zeros(1, dtype=torch.int32, device=dev) if status is None else status
    if workspace is None:
        workspace = torch.zeros(max(sb_fuse_project_workspace_bytes(n_starts, block_k, d, d_out, q_term_valid), 256),
                                dtype=torch.uint8, device=dev)
    rc = load().sb_fuse_project(_ptr(c, torch.bfloat16), _ptr(e, torch.bfloat16), _ptr(q, torch.bfloat16),
                                _ptr(gain_c, torch.float32), _ptr(gain_e, torch.float32), _ptr(gain_q, torch.float32),
                                C.c_float(eps), _ptr(w, torch.bfloat16), C.c_int32(n_starts), C.c_int32(block_k),
                                C.c_int32(d), C.c_int32(d_out), _ptr(q_term, torch.float32),
                                C.c_int32(1 if q_term_valid else 0), _ptr(out, torch.bfloat16), _ptr(workspace),
                                C.c_size_t(workspace.numel()), _ptr(status, torch.int32), _stream())
    _check(rc, "sb_fuse_project")
    return out, status


SB_STATIC_SCRATCH_BYTES = 256 * 1024


def sb_verify_accept_static(logits, node_offsets, parent, tok, max_depth, out, *, vocab=None):
    """sb_verify_accept without a workspace, for callers that cannot allocate device memory: the
    library's own fixed scratch array is used (at most SB_STATIC_SCRATCH_BYTES of partials, else
    SB_ERR_WORKSPACE).  `out` must hold the preallocated result tensors (amax, accept_len,
    path_nodes, out_tokens, bonus, status): nothing is allocated here either.  Calls that may
    overlap on the GPU share that array and must be serialised by the caller."""
    total, stride = logits.shape
    vocab = stride if vocab is None else vocab
    batch = node_offsets.numel() - 1
    dt = {torch.bfloat16: SB_BF16, torch.float32: SB_F32}[logits.dtype]
    rc = load().sb_verify_accept_static(
        _ptr(logits), C.c_int(dt), C.c_int64(stride), C.c_int32(vocab), C.c_int32(batch), C.c_int32(total),
        _ptr(node_offsets, torch.int32), _ptr(parent, torch.int32), _ptr(tok, torch.int32),
        C.c_int32(max_depth), _ptr(out["amax"]), _ptr(out["accept_len"]), _ptr(out["path_nodes"]),
        _ptr(out["out_tokens"]), _ptr(out["bonus"]), _ptr(out["status"]), _stream())
    _check(rc, "sb_verify_accept_static")
    return out


def sb_kv_compact(tb: TreeBatch, n_layers, layer_stride_elems, path_nodes, accept_len, max_depth,
                  new_len=None, status=None):
    """In-place compaction of tb.k_cache / tb.v_cache (layer 0 of n_layers).  -> (new_len, status)."""
    batch = tb.prefix_len.numel()
    dev = tb.prefix_len.device
    new_len = torch.empty(batch, dtype=torch.int32, device=dev) if new_len is None else new_len
    status = torch.empty(batch, dtype=torch.int32, device=dev) if status is None else status
    s = tb.c_struct()
    rc = load().sb_kv_compact(C.byref(s), C.c_int32(n_layers), C.c_int64(layer_stride_elems),
                              _ptr(path_nodes, torch.int32), _ptr(accept_len, torch.int32),
                              C.c_int32(max_depth), _ptr(new_len, torch.int32),
                              _ptr(status, torch.int32), _stream())
    _check(rc, "sb_kv_compact")
    return new_len, status


def sb_path_rows(node_offsets, node_row, path_nodes, accept_len, max_depth, path_rows=None, status=None,
                 row_begin=None):
    """The accepted path in the drafter's row numbering: -> (path_rows int32 [B, max_depth+1], status [B])."""
    batch = node_offsets.numel() - 1
    dev = node_row.device
    if path_rows is None:
        path_rows = torch.empty((batch, max_depth + 1), dtype=torch.int32, device=dev)
    status = torch.empty(batch, dtype=torch.int32, device=dev) if status is None else status
    rc = load().sb_path_rows(C.c_int32(batch), _ptr(node_offsets, torch.int32), _ptr(node_row, torch.int32),
                             _ptr(row_begin, torch.int32), _ptr(path_nodes, torch.int32),
                             _ptr(accept_len, torch.int32), C.c_int32(max_depth), _ptr(path_rows, torch.int32),
                             _ptr(status, torch.int32), _stream())
    _check(rc, "sb_path_rows")
    return path_rows, status


def sb_tree_expand_workspace_bytes(n_rows: int, vocab: int) -> int:
    return int(load().sb_tree_expand_workspace_bytes(C.c_int32(n_rows), C.c_int32(vocab)))


def sb_tree_expand(scores, block_k, bucket, bmap, start_parent, node_budget, tree, *, vocab=None,
                   workspace=None, topk_tok=None, topk_val=None, status=None, features=None, child_row=None,
                   row_base=0):
    """scores fp32 [R, stride]; bucket uint8 [R]; bmap: 4 host ints; tree: dict of int32 device
    tensors n_nodes [1], tok, parent, depth, node_row, node_rank (capacity node_budget), updated
    in place.  -> (topk_tok [R,16], topk_val [R,16], status [1]).
    features fp32 [R, 15]: also filled (sb_tree_expand_features: one pass over the scores for both);
    the workspace must then hold sb_rank_features_workspace_bytes.  With features, child_row int32
    [node_budget] (initialised to -1 by the caller) receives row_base + row for the nodes whose children a row
    of this call proposes."""
    n_rows, stride = scores.shape
    vocab = stride if vocab is None else vocab
    dev = scores.device
    topk_tok = torch.empty((n_rows, SB_KMAX), dtype=torch.int32, device=dev) if topk_tok is None else topk_tok
    topk_val = torch.empty((n_rows, SB_KMAX), dtype=torch.float32, device=dev) if topk_val is None else topk_val
    status = torch.empty(1, dtype=torch.int32, device=dev) if status is None else status
    lib = load()
    if workspace is None:
        need = (sb_tree_expand_workspace_bytes if features is None else sb_rank_features_workspace_bytes)(n_rows, vocab)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    bm = (C.c_int32 * 4)(*[int(x) for x in bmap])
    head = (_ptr(scores, torch.float32), C.c_int64(stride), C.c_int32(n_rows),
            C.c_int32(vocab), C.c_int32(block_k), _ptr(bucket, torch.uint8), bm,
            _ptr(start_parent, torch.int32), C.c_int32(node_budget),
            _ptr(tree["n_nodes"], torch.int32), _ptr(tree["tok"], torch.int32),
            _ptr(tree["parent"], torch.int32), _ptr(tree["depth"], torch.int32),
            _ptr(tree["node_row"], torch.int32), _ptr(tree["node_rank"], torch.int32),
            _ptr(topk_tok, torch.int32), _ptr(topk_val, torch.float32))
    tail = (_ptr(workspace), C.c_size_t(workspace.numel()), _ptr(status, torch.int32), _stream())
    if features is None:
        _check(lib.sb_tree_expand(*head, *tail), "sb_tree_expand")
    else:
        _check(lib.sb_tree_expand_features(*head, _ptr(features, torch.float32), _ptr(child_row, torch.int32),
                                           C.c_int32(row_base), *tail), "sb_tree_expand_features")
    return topk_tok, topk_val, status


# ---- a KV cache in 8 bits ----------------------------------------------------------------------------------------------

class _QuantCache(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("scale_block", C.c_int32),
        ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
        ("page_size", C.c_int32), ("max_pages", C.c_int32), ("kv_capacity", C.c_int64), ("num_pages", C.c_int32),
        ("n_layers", C.c_int32), ("codes_layer_stride", C.c_int64), ("scale_layer_stride", C.c_int64),
        ("page_table", C.c_void_p),
    ]


class _QuantTree(C.Structure):
    _fields_ = [
        ("n_q_heads", C.c_int32), ("total_nodes", C.c_int32), ("max_nodes", C.c_int32), ("max_prefix", C.c_int32),
        ("prefix_len", C.c_void_p), ("node_offsets", C.c_void_p), ("parent", C.c_void_p),
    ]


class _PagePool(C.Structure):
    _fields_ = [
        ("num_pages", C.c_int32), ("page_size", C.c_int32), ("n_slots", C.c_int32), ("max_pages", C.c_int32),
        ("page_table", C.c_void_p), ("held", C.c_void_p), ("refs", C.c_void_p),
    ]


class _PageArray(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_bytes", C.c_int64), ("layer_stride", C.c_int64)]


def _refuse(t, dtype, device, numel):
    if t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"expected a tensor on {'the CPU' if device < 0 else f'cuda:{device}'}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    raise ValueError(f"expected {numel} elements, got {tuple(t.shape)}")


def _addr(t, dtype, device, numel=None):
    """Address of a contiguous tensor of this type on this device (its index, -1 for the CPU); None: a null pointer."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous() or (numel is not None and t.numel() != numel):
        _refuse(t, dtype, device, numel)
    return t.data_ptr()


def _cuda_device(t):
    """Index of the tensor's device, which has to be the current one: the library enqueues on the current device's stream."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("expected a CUDA tensor")
    if dev != torch.cuda.current_device():
        raise ValueError(f"tensors are on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return dev


# The current stream's handle without building a Stream object for every call, where torch has that.
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


@dataclass(frozen=True)
class QuantCache:
    """A KV cache held as e4m3 codes with one fp32 scale for each block of scale_block tokens and KV head; mirrors the C
    struct sb_quant_cache.  k_codes / v_codes: uint8 or float8_e4m3fn, contiguous, [(layers,) batch, capacity, Hkv, D], or
    paged [(layers,) pages, page_size, Hkv, D] with page_table int32 [batch, max_pages].  k_scale / v_scale: fp32
    [(layers,) batch, capacity / scale_block, Hkv] or [(layers,) pages, page_size / scale_block, Hkv].  The tensors'
    contents may change between calls; another tensor takes another QuantCache."""
    k_codes: torch.Tensor
    v_codes: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    n_kv_heads: int
    head_dim: int
    scale_block: int
    page_size: int = 0
    page_table: Optional[torch.Tensor] = None
    n_layers: int = 1

    def __post_init__(self):
        s = _QuantCache()
        dev = self.k_codes.get_device()
        lead = self.k_codes.shape[:-2]
        if self.k_codes.dim() != (4 if self.n_layers == 1 and self.k_codes.dim() == 4 else 5):
            raise ValueError("codes must be [(layers,) rows, tokens, n_kv_heads, head_dim]")
        if tuple(self.k_codes.shape[-2:]) != (self.n_kv_heads, self.head_dim) or self.v_codes.shape != self.k_codes.shape:
            raise ValueError("k_codes and v_codes must both end in [n_kv_heads, head_dim]")
        if len(lead) == 3 and lead[0] != self.n_layers:
            raise ValueError("the codes' first dimension must be n_layers")
        rows, tokens = lead[-2:]
        if self.scale_block < 1 or tokens % self.scale_block:
            raise ValueError("the tokens of a page (or of a contiguous sequence) must be a multiple of scale_block")
        scales = self.n_layers * rows * (tokens // self.scale_block) * self.n_kv_heads
        for name, t in (("k_codes", self.k_codes), ("v_codes", self.v_codes)):
            if t.dtype not in (torch.uint8, torch.float8_e4m3fn):
                raise TypeError(f"{name}: expected uint8 or float8_e4m3fn, got {t.dtype}")
            setattr(s, name, _addr(t, t.dtype, dev))
        s.k_scale = _addr(self.k_scale, torch.float32, dev, scales)
        s.v_scale = _addr(self.v_scale, torch.float32, dev, scales)
        s.n_kv_heads, s.head_dim, s.scale_block = self.n_kv_heads, self.head_dim, self.scale_block
        s.page_size, s.n_layers = self.page_size, self.n_layers
        s.codes_layer_stride = self.k_codes.numel() // self.n_layers
        s.scale_layer_stride = scales // self.n_layers
        if self.page_size:
            if tokens != self.page_size or self.page_table is None or self.page_table.dim() != 2:
                raise ValueError("a paged cache needs codes of page_size tokens a page and a page_table [batch, max_pages]")
            s.batch, s.max_pages = self.page_table.shape
            s.num_pages, s.kv_capacity = rows, 0
            s.page_table = _addr(self.page_table, torch.int32, dev)
        else:
            s.batch, s.kv_capacity, s.max_pages, s.num_pages = rows, tokens, 0, 0
        object.__setattr__(self, "c_struct", s)
        object.__setattr__(self, "c_ref", C.addressof(s))
        object.__setattr__(self, "batch", int(s.batch))
        object.__setattr__(self, "device", dev)


@dataclass(frozen=True)
class QuantTree:
    """The ragged batch of draft trees that attends to a QuantCache; mirrors the C struct sb_quant_tree."""
    n_q_heads: int
    prefix_len: torch.Tensor     # int32 [B]
    node_offsets: torch.Tensor   # int32 [B+1]
    parent: torch.Tensor         # int32 [total_nodes]
    max_nodes: int
    max_prefix: int

    def __post_init__(self):
        s = _QuantTree()
        dev = self.prefix_len.get_device()
        s.n_q_heads, s.total_nodes = self.n_q_heads, self.parent.numel()
        s.max_nodes, s.max_prefix = self.max_nodes, self.max_prefix
        s.prefix_len = _addr(self.prefix_len, torch.int32, dev)
        s.node_offsets = _addr(self.node_offsets, torch.int32, dev, self.prefix_len.numel() + 1)
        s.parent = _addr(self.parent, torch.int32, dev)
        object.__setattr__(self, "c_struct", s)
        object.__setattr__(self, "c_ref", C.addressof(s))
        object.__setattr__(self, "device", dev)
        object.__setattr__(self, "batch", self.prefix_len.numel())
        object.__setattr__(self, "total_nodes", self.parent.numel())


def _rows_of(t, heads, dim, device, what, dims=3):
    """(address, elements between rows) of bf16 rows [..., heads, dim] whose rows are contiguous inside: a whole tensor or
    a slice of a fused projection, of `dims` dimensions (the caller sees to those before the rows)."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{what}: expected torch.bfloat16, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on cuda:{device}, got {t.device}")
    shape = t.shape
    if len(shape) < 3 or shape[-2] != heads or shape[-1] != dim:
        raise ValueError(f"{what}: expected rows of [{heads}, {dim}], got {tuple(shape)}")
    if t.is_contiguous():
        return t.data_ptr(), heads * dim
    if len(shape) != dims:
        raise ValueError(f"{what}: expected strided rows in {dims} dimensions, got {tuple(shape)}")
    stride = t.stride()
    if stride[-1] != 1 or (heads > 1 and stride[-2] != dim):
        raise ValueError(f"{what}: expected rows that are contiguous inside, got strides {stride}")
    if shape[-3] <= 1:
        return t.data_ptr(), heads * dim
    if stride[-3] < heads * dim:  # an expanded tensor: 0 means "one row behind the other" to the library, past the tensor's end
        raise ValueError(f"{what}: expected rows that do not overlap, got strides {stride}")
    return t.data_ptr(), stride[-3]


def sb_tree_attention_quant_workspace_bytes(kv: QuantCache, tree: QuantTree, total_q: int, *, num_splits: int = 0,
                                            window: int = 0, sinks: int = 0) -> int:
    return int(load().sb_tree_attention_quant_workspace_bytes(kv.c_ref, tree.c_ref, total_q, window, sinks, num_splits))


def sb_tree_attention_quant(kv: QuantCache, tree: QuantTree, q, k_nodes, v_nodes, *, layer=0, window=0, sinks=0, out=None,
                            lse=None, q_node_begin=None, q_offsets=None, scale=0.0, num_splits=0, workspace=None,
                            status=None, want_lse=True):
    """q bf16 [total_q, Hq, D], k_nodes / v_nodes bf16 [total_nodes, Hkv, D] (rows may be strided) over the 8-bit prefix ->
    (out bf16 [total_q, Hq, D], lse fp32 [total_q, Hq] or None, status [B]).  window > 0: a node at position x sees
    positions above x - window and the first `sinks`."""
    dev = _cuda_device(q)
    total_q = q.shape[0]
    Hq, D, B = tree.n_q_heads, kv.head_dim, kv.batch
    if tree.batch != B:
        raise ValueError("the tree batch and the cache have different numbers of sequences")
    if kv.device != dev or tree.device != dev:
        raise ValueError(f"cache, tree and q must all be on cuda:{dev}")
    q_ptr, q_stride = _rows_of(q, Hq, D, dev, "q")
    total = tree.total_nodes
    if k_nodes.shape[0] != total or v_nodes.shape[0] != total:
        raise ValueError(f"k_nodes and v_nodes must have {total} rows")
    k_ptr, k_stride = _rows_of(k_nodes, kv.n_kv_heads, D, dev, "k_nodes")
    v_ptr, v_stride = _rows_of(v_nodes, kv.n_kv_heads, D, dev, "v_nodes")
    if k_stride != v_stride:
        raise ValueError("k_nodes and v_nodes must have the same stride between rows")
    if q_node_begin is None and q_offsets is None and total_q != total:
        raise ValueError(f"q must have one row for each of the {total} nodes, or q_offsets must say where its rows are")
    out = torch.empty((total_q, Hq, D), dtype=torch.bfloat16, device=dev) if out is None else out
    if lse is None and want_lse:
        lse = torch.empty((total_q, Hq), dtype=torch.float32, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev) if status is None else status
    lib = load()
    if workspace is None:
        need = lib.sb_tree_attention_quant_workspace_bytes(kv.c_ref, tree.c_ref, total_q, window, sinks, num_splits)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    rc = lib.sb_tree_attention_quant(
        kv.c_ref, layer, tree.c_ref, k_ptr, v_ptr, k_stride, _addr(q_node_begin, torch.int32, dev, B),
        _addr(q_offsets, torch.int32, dev, B), total_q, q_ptr, q_stride, _addr(out, torch.bfloat16, dev, total_q * Hq * D),
        _addr(lse, torch.float32, dev, total_q * Hq), scale, window, sinks, num_splits, _addr(workspace, torch.uint8, dev),
        workspace.numel(), _addr(status, torch.int32, dev, B), _stream_of(dev))
    _check(rc, "sb_tree_attention_quant")
    return out, lse, status


def sb_kv_append_quant(kv: QuantCache, k_rows, v_rows, row_offsets, length, *, max_rows, path_nodes=None, accept_len=None,
                       max_depth=0, new_len=None, status=None):
    """Appends bf16 rows k_rows / v_rows [(layers,) rows, Hkv, D] to the cache behind length int32 [B]: rows
    row_offsets[b] .. row_offsets[b+1] - 1, or with path_nodes and accept_len (as sb_verify_accept leaves them) the accepted
    path's rows.  max_rows bounds the rows of a sequence.  -> (new_len [B], status [B])."""
    dev = _cuda_device(k_rows)
    if kv.device != dev:
        raise ValueError(f"cache and rows must both be on cuda:{dev}")
    B = kv.batch
    if k_rows.shape != v_rows.shape or k_rows.stride() != v_rows.stride():
        raise ValueError("k_rows and v_rows must have the same shape and strides")
    if k_rows.dim() == 4:
        if k_rows.shape[0] != kv.n_layers:
            raise ValueError(f"the rows' first dimension must be the cache's {kv.n_layers} layers")
        layer_stride = k_rows.stride(0) if kv.n_layers > 1 else 0
    elif k_rows.dim() == 3 and kv.n_layers == 1:
        layer_stride = 0
    else:
        raise ValueError("rows must be [layers, rows, n_kv_heads, head_dim]")
    k_ptr, stride = _rows_of(k_rows, kv.n_kv_heads, kv.head_dim, dev, "k_rows", k_rows.dim())
    v_ptr, _ = _rows_of(v_rows, kv.n_kv_heads, kv.head_dim, dev, "v_rows", k_rows.dim())
    new_len = torch.empty(B, dtype=torch.int32, device=dev) if new_len is None else new_len
    status = torch.empty(B, dtype=torch.int32, device=dev) if status is None else status
    rc = load().sb_kv_append_quant(
        kv.c_ref, k_ptr, v_ptr, stride, layer_stride, _addr(row_offsets, torch.int32, dev, B + 1), k_rows.shape[-3],
        _addr(path_nodes, torch.int32, dev, B * (max_depth + 1)), _addr(accept_len, torch.int32, dev, B), max_depth, max_rows,
        _addr(length, torch.int32, dev, B), _addr(new_len, torch.int32, dev, B), _addr(status, torch.int32, dev, B),
        _stream_of(dev))
    _check(rc, "sb_kv_append_quant")
    return new_len, status


# ---- pages of a cache ------------------------------------------------------------------------------------------------

@dataclass(frozen=True)
class PagePool:
    """Bookkeeping of a paged cache (int32 device tensors); mirrors the C struct sb_page_pool.  page_table [slots,
    max_pages] (-1 behind a slot's pages), held [slots], refs [num_pages] (0 = free)."""
    page_size: int
    page_table: torch.Tensor
    held: torch.Tensor
    refs: torch.Tensor

    def __post_init__(self):
        s = _PagePool()
        dev = self.page_table.get_device()
        if self.page_table.dim() != 2:
            raise ValueError("page_table must be [slots, max_pages]")
        s.page_size, s.num_pages = self.page_size, self.refs.numel()
        s.n_slots, s.max_pages = self.page_table.shape
        s.page_table = _addr(self.page_table, torch.int32, dev)
        s.held = _addr(self.held, torch.int32, dev, s.n_slots)
        s.refs = _addr(self.refs, torch.int32, dev)
        object.__setattr__(self, "c_struct", s)
        object.__setattr__(self, "c_ref", C.addressof(s))
        object.__setattr__(self, "device", dev)

    @classmethod
    def empty(cls, n_slots, max_pages, num_pages, page_size, device="cuda"):
        """A pool of free pages."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(page_size, torch.full((n_slots, max_pages), -1, **i32), torch.zeros(n_slots, **i32), torch.zeros(num_pages, **i32))


@dataclass(frozen=True)
class PageCopies:
    """The (source, destination) page pairs that sb_pages_reserve / sb_pages_compact leave for sb_pages_copy: src, dst
    int32 [room], the pairs first, count[0] of them; then -1, after sb_pages_reserve up to the length of its list."""
    src: torch.Tensor
    dst: torch.Tensor
    count: torch.Tensor

    @classmethod
    def empty(cls, room, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((room,), -1, **i32), torch.full((room,), -1, **i32), torch.zeros(1, **i32))


@dataclass(frozen=True)
class PageArrays:
    """The arrays that a page id indexes, each [pages, ...] or [layers, pages, ...], contiguous: K and V codes and scales of
    an 8-bit cache, or K and V of a bf16 one."""
    tensors: list
    n_layers: int
    num_pages: int

    def __post_init__(self):
        arr = (_PageArray * len(self.tensors))()
        for a, t in zip(arr, self.tensors):
            lead = t.shape[:2] if self.n_layers > 1 or t.shape[0] != self.num_pages else (1, t.shape[0])
            if tuple(lead) != (self.n_layers, self.num_pages):
                raise ValueError(f"expected [{self.n_layers}, {self.num_pages}, ...] (or without layers), got {tuple(t.shape)}")
            layer = t.numel() // self.n_layers * t.element_size()
            a.base, a.page_bytes, a.layer_stride = _addr(t, t.dtype, self.tensors[0].get_device()), layer // self.num_pages, layer
        object.__setattr__(self, "c_array", arr)
        object.__setattr__(self, "c_ref", C.addressof(arr))
        object.__setattr__(self, "device", self.tensors[0].get_device())


def sb_pages_workspace_bytes(pool: PagePool, n: int) -> int:
    return int(load().sb_pages_workspace_bytes(pool.c_ref, n))


def _pages_call(pool, n, workspace, status, entries):
    dev = _cuda_device(pool.page_table)
    if workspace is None:
        workspace = torch.empty(max(sb_pages_workspace_bytes(pool, n), 256), dtype=torch.uint8, device=dev)
    status = torch.empty(entries, dtype=torch.int32, device=dev) if status is None else status
    return dev, (_addr(workspace, torch.uint8, dev), workspace.numel(), _addr(status, torch.int32, dev, entries), _stream_of(dev)), status, workspace


def sb_pages_fork(pool: PagePool, src, dst, length, *, workspace=None, status=None):
    """Slots dst (int32 [n], empty) share the pages of slots src that hold their first `length` positions.  -> status [n]."""
    n = src.numel()
    dev, tail, status, workspace = _pages_call(pool, n, workspace, status, n)
    rc = load().sb_pages_fork(pool.c_ref, n, _addr(src, torch.int32, dev), _addr(dst, torch.int32, dev, n),
                              _addr(length, torch.int32, dev, n), *tail)
    _check(rc, "sb_pages_fork")
    return status


def sb_pages_reserve(pool: PagePool, slots, keep_len, new_len, copies: PageCopies, *, workspace=None, status=None):
    """Makes positions [keep_len, new_len) of the slots writable: adds pages, and replaces shared ones; what has to be copied
    goes to `copies` (room for n pairs).  -> status [n]."""
    n = slots.numel()
    dev, tail, status, workspace = _pages_call(pool, n, workspace, status, n)
    if copies.src.numel() < n:
        raise ValueError(f"copies needs room for {n} pairs")
    rc = load().sb_pages_reserve(pool.c_ref, n, _addr(slots, torch.int32, dev), _addr(keep_len, torch.int32, dev, n),
                                 _addr(new_len, torch.int32, dev, n), _addr(copies.src, torch.int32, dev),
                                 _addr(copies.dst, torch.int32, dev, copies.src.numel()), _addr(copies.count, torch.int32, dev, 1), *tail)
    _check(rc, "sb_pages_reserve")
    return status


def sb_pages_release(pool: PagePool, slots, keep_len, *, workspace=None, status=None):
    """The slots keep the pages of their first keep_len positions.  -> status [n]."""
    n = slots.numel()
    dev, tail, status, workspace = _pages_call(pool, n, workspace, status, n)
    rc = load().sb_pages_release(pool.c_ref, n, _addr(slots, torch.int32, dev), _addr(keep_len, torch.int32, dev, n), *tail)
    _check(rc, "sb_pages_release")
    return status


def sb_pages_compact(pool: PagePool, copies: PageCopies, *, n_used=None, workspace=None, status=None):
    """Moves the pages in use to the front of the pool; `copies` (room for num_pages // 2 pairs) says what sb_pages_copy
    has to move.  -> status [1]."""
    dev, tail, status, workspace = _pages_call(pool, 0, workspace, status, 1)
    rc = load().sb_pages_compact(pool.c_ref, _addr(copies.src, torch.int32, dev), _addr(copies.dst, torch.int32, dev, copies.src.numel()),
                                 copies.src.numel(), _addr(copies.count, torch.int32, dev, 1), _addr(n_used, torch.int32, dev, 1), *tail)
    _check(rc, "sb_pages_compact")
    return status


def sb_pages_copy(arrays: PageArrays, copies: PageCopies):
    """Copies the contents of the pages in `copies`, every layer of every array, in one launch."""
    dev = _cuda_device(copies.src)
    if arrays.device != dev:
        raise ValueError(f"expected arrays on cuda:{dev}")
    rc = load().sb_pages_copy(arrays.c_ref, len(arrays.tensors), arrays.n_layers, arrays.num_pages, _addr(copies.src, torch.int32, dev),
                              _addr(copies.dst, torch.int32, dev, copies.src.numel()), _addr(copies.count, torch.int32, dev, 1),
                              copies.src.numel(), _stream_of(dev))
    _check(rc, "sb_pages_copy")


# ---- hooks of the test and checked builds (include/specblock_test.h); use inside build_variant(...) ----

def sb_test_wait_expires(limit_ns: int):
    """Test build: lets a bounded device wait run out.  -> (status int32[1], elapsed_ns int64[2]) tensors."""
    lib = load()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    elapsed = torch.zeros(2, dtype=torch.int64, device="cuda")
    lib.sb_test_wait_expires.restype = C.c_int
    _check(lib.sb_test_wait_expires(C.c_int64(limit_ns), _ptr(status), _ptr(elapsed), _stream()), "sb_test_wait_expires")
    return status, elapsed


def sb_checked_violations() -> int:
    """Checked build: accesses refused since the last call (synchronises the device, clears the counter)."""
    lib = load()
    lib.sb_checked_violations.restype = C.c_int
    n = C.c_int64(-1)
    _check(lib.sb_checked_violations(C.byref(n)), "sb_checked_violations")
    return int(n.value)


def sb_checked_selftest():
    """Checked build: one refused access on purpose.  -> status int32[2] tensor."""
    lib = load()
    lib.sb_checked_selftest.restype = C.c_int
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    _check(lib.sb_checked_selftest(_ptr(status), _stream()), "sb_checked_selftest")
    return status
