"""Python binding of the C-ABI library (include/oomb.h): argument marshalling
only.  Torch supplies device memory and the stream; every step of the path runs
in the library's HIP kernels.  Function names mirror the C entry points.

The calls of a loop over chunks go through the native module _binding (csrc/binding.cpp), which checks the tensors against
the descriptor and calls the library; it answers -1 if something does not fit, and the checks here then say what.
The other entry points are marshalled with ctypes."""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liboomb.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_LAUNCH, ERR_OUT_OF_PAGES, ERR_SCRATCH_LIMIT = range(7)
NOALLOC_SCRATCH_BYTES = 4 << 20
F32, BF16 = 0, 1
OP_SCORE_TOPK, OP_ATTN_FWD, OP_ATTN_BWD, OP_VOTE_TOPK, OP_ATTN_FWD_QP, OP_ATTN_BWD_QP, \
    OP_CHECK_INPUTS = range(7)

EXPORTS = ["oomb_workspace_bytes", "oomb_page_score_topk", "oomb_paged_attn_fwd",
           "oomb_paged_attn_bwd", "oomb_status_string", "oomb_version", "oomb_profile_enable",
           "oomb_profile_reset", "oomb_profile_count", "oomb_profile_read", "oomb_calibrate",
           "oomb_kv_append", "oomb_page_means", "oomb_page_score_topk_cached", "oomb_local_page_list",
           "oomb_page_pool_reset", "oomb_page_pool_alloc", "oomb_page_pool_release",
           "oomb_paged_attn_fwd_qp", "oomb_paged_attn_bwd_qp", "oomb_page_vote_topk",
           "oomb_offload_plan", "oomb_offload_fetch", "oomb_offload_writeback", "oomb_check_inputs",
           "oomb_page_score_topk_noalloc", "oomb_kv_append_rope", "oomb_kv_append_rope_bwd",
           "oomb_kvq_append_rope", "oomb_kvq_read", "oomb_kvq_workspace_bytes", "oomb_paged_attn_fwd_kvq",
           "oomb_rows_workspace_bytes", "oomb_paged_attn_fwd_rows", "oomb_page_fork_workspace_bytes", "oomb_page_fork",
           "oomb_page_compact_workspace_bytes", "oomb_page_compact", "oomb_page_copy", "oomb_beam_workspace_bytes", "oomb_beam_topk"]


class AttnDesc(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("chunk_len", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("ctx_len", ctypes.c_int64),
                ("pool_page_stride", ctypes.c_int64), ("pool_head_stride", ctypes.c_int64),
                ("pool_tok_stride", ctypes.c_int64),
                ("q_tok_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("num_phys_pages", ctypes.c_int64)]


class RowsDesc(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("max_len", ctypes.c_int64), ("table_stride", ctypes.c_int64), ("num_phys_pages", ctypes.c_int64),
                ("pool_page_stride", ctypes.c_int64), ("pool_head_stride", ctypes.c_int64),
                ("pool_tok_stride", ctypes.c_int64)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("tok_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Seqs(ctypes.Structure):
    _fields_ = [("page_tables", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("row_starts", ctypes.c_void_p)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("n_pos", ctypes.c_int64),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class PagesDesc(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_out", ctypes.c_int32), ("page_size", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("table_cols", ctypes.c_int64), ("table_stride", ctypes.c_int64), ("out_cols", ctypes.c_int64), ("out_stride", ctypes.c_int64),
                ("num_phys_pages", ctypes.c_int64)]


class CopyDesc(ctypes.Structure):
    _fields_ = [("n_pools", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("page_size", ctypes.c_int32), ("row_bytes", ctypes.c_int32),
                ("num_phys_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("tok_stride", ctypes.c_int64),
                ("max_copies", ctypes.c_int64)]


class BeamDesc(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int32), ("n_beams", ctypes.c_int32), ("vocab", ctypes.c_int32), ("n_out", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("pad_token", ctypes.c_int32), ("row_stride", ctypes.c_int64)]


class OombError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib():
    """The loaded C-ABI library.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2602_02108_amd.build "
                               "or __graft_entry__.build())")
        l = ctypes.CDLL(LIB_PATH)
        vp, i32, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        dp = ctypes.POINTER(AttnDesc)
        l.oomb_workspace_bytes.restype = u64
        l.oomb_workspace_bytes.argtypes = [dp, i32, i32]
        l.oomb_page_score_topk.restype = i32
        l.oomb_page_score_topk.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp, vp, u64, vp]
        l.oomb_page_score_topk_noalloc.restype = i32
        l.oomb_page_score_topk_noalloc.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp, vp]
        l.oomb_paged_attn_fwd.restype = i32
        l.oomb_paged_attn_fwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, u64, vp]
        l.oomb_paged_attn_bwd.restype = i32
        l.oomb_paged_attn_bwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, u64, vp]
        l.oomb_paged_attn_fwd_qp.restype = i32
        l.oomb_paged_attn_fwd_qp.argtypes = l.oomb_paged_attn_fwd.argtypes
        l.oomb_paged_attn_bwd_qp.restype = i32
        l.oomb_paged_attn_bwd_qp.argtypes = l.oomb_paged_attn_bwd.argtypes
        l.oomb_page_vote_topk.restype = i32
        l.oomb_page_vote_topk.argtypes = [dp, vp, vp, i32, vp, vp, vp, vp, u64, vp]
        l.oomb_offload_plan.restype = i32
        l.oomb_offload_plan.argtypes = [dp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]
        l.oomb_offload_fetch.restype = i32
        l.oomb_offload_fetch.argtypes = [dp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
        l.oomb_offload_writeback.restype = i32
        l.oomb_offload_writeback.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
        l.oomb_check_inputs.restype = i32
        l.oomb_check_inputs.argtypes = [dp, vp, vp, vp, i32, i32, vp, vp, u64, vp]
        l.oomb_status_string.restype = ctypes.c_char_p
        l.oomb_status_string.argtypes = [i32]
        l.oomb_version.restype = i32
        l.oomb_profile_enable.restype = None
        l.oomb_profile_enable.argtypes = [i32]
        l.oomb_profile_reset.restype = None
        l.oomb_profile_count.restype = i32
        l.oomb_profile_read.restype = i32
        l.oomb_profile_read.argtypes = [i32, ctypes.c_char_p, i32, ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_int64)]
        i64, fp = ctypes.c_int64, ctypes.c_void_p
        l.oomb_kv_append.restype = i32
        l.oomb_kv_append.argtypes = [dp, vp, vp, vp, vp, vp, fp, vp]
        l.oomb_page_means.restype = i32
        l.oomb_page_means.argtypes = [dp, vp, vp, i64, i64, fp, vp]
        l.oomb_page_score_topk_cached.restype = i32
        l.oomb_page_score_topk_cached.argtypes = [dp, vp, fp, i32, vp, vp, vp, vp, u64, vp]
        l.oomb_local_page_list.restype = i32
        l.oomb_local_page_list.argtypes = [dp, i32, vp, vp, vp]
        l.oomb_page_pool_reset.restype = i32
        l.oomb_page_pool_reset.argtypes = [i64, vp, ctypes.POINTER(i64)]
        l.oomb_page_pool_alloc.restype = i32
        l.oomb_page_pool_alloc.argtypes = [vp, ctypes.POINTER(i64), i64, vp]
        l.oomb_page_pool_release.restype = i32
        l.oomb_page_pool_release.argtypes = [i64, vp, ctypes.POINTER(i64), vp, i64]
        l.oomb_calibrate.restype = i32
        l.oomb_calibrate.argtypes = [i32, vp, u64, ctypes.POINTER(ctypes.c_double), vp]
        rd, rw, sq, rp = (ctypes.POINTER(t) for t in (RowsDesc, Rows, Seqs, RopeDesc))
        for f in (l.oomb_kv_append_rope, l.oomb_kvq_append_rope):
            f.restype = i32
            f.argtypes = [rd, sq, rp, rw, rw, rw, rw, vp, vp, vp, vp]
        l.oomb_kv_append_rope_bwd.restype = i32
        l.oomb_kv_append_rope_bwd.argtypes = [rd, sq, rp, rw, rw, vp, vp, i32, rw, rw, vp]
        l.oomb_kvq_read.restype = i32
        l.oomb_kvq_read.argtypes = [rd, sq, vp, vp, rw, rw, vp]
        l.oomb_kvq_workspace_bytes.restype = u64
        l.oomb_kvq_workspace_bytes.argtypes = [rd, i32]
        l.oomb_paged_attn_fwd_kvq.restype = i32
        l.oomb_paged_attn_fwd_kvq.argtypes = [rd, sq, rw, vp, vp, vp, vp, i32, rw, vp, vp, u64, vp]
        l.oomb_rows_workspace_bytes.restype = u64
        l.oomb_rows_workspace_bytes.argtypes = [rd, i32]
        l.oomb_paged_attn_fwd_rows.restype = i32
        l.oomb_paged_attn_fwd_rows.argtypes = l.oomb_paged_attn_fwd_kvq.argtypes
        pd, cd, bd = (ctypes.POINTER(t) for t in (PagesDesc, CopyDesc, BeamDesc))
        l.oomb_page_fork_workspace_bytes.restype = u64
        l.oomb_page_fork_workspace_bytes.argtypes = [i32, i32, i64]
        l.oomb_page_fork.restype = i32
        l.oomb_page_fork.argtypes = [pd] + [vp] * 11 + [u64, vp]
        l.oomb_page_compact_workspace_bytes.restype = u64
        l.oomb_page_compact_workspace_bytes.argtypes = [i64]
        l.oomb_page_compact.restype = i32
        l.oomb_page_compact.argtypes = [pd] + [vp] * 6 + [i64, vp, vp, vp, u64, vp]
        l.oomb_page_copy.restype = i32
        l.oomb_page_copy.argtypes = [cd, vp, vp, vp, vp]
        l.oomb_beam_workspace_bytes.restype = u64
        l.oomb_beam_workspace_bytes.argtypes = [bd]
        l.oomb_beam_topk.restype = i32
        l.oomb_beam_topk.argtypes = [bd] + [vp] * 7 + [u64, vp]
        _lib = l
    return _lib


_nb = None


def _native():
    """The native module; like the library it has no fallback."""
    global _nb
    if _nb is None:
        lib()
        from . import _binding
        _nb = _binding
    return _nb


def _refused(where: str):
    """The native module found a tensor that does not fit, and no check here said which."""
    return OombError(ERR_INVALID_ARG, f"{where}: an argument is no device tensor or does not fit the descriptor")


def _no_workspace(desc, top_k: int, op: int) -> bool:
    """Whether the descriptor is one that oomb_workspace_bytes refuses, which takes precedence over the status of the call."""
    return workspace_bytes(desc, top_k, op) == 0 and (op == OP_SCORE_TOPK or top_k >= 0 or workspace_bytes(desc, -1, op) == 0)


def status_string(status: int) -> str:
    return lib().oomb_status_string(int(status)).decode()


def version() -> int:
    return int(lib().oomb_version())


def _dt(t: torch.dtype) -> int:
    if t == torch.float32:
        return F32
    if t == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t}")


def make_desc(q: torch.Tensor, k_pool: torch.Tensor, ctx_len: int, sm_scale: float,
              grad_dtype: torch.dtype = torch.float32) -> AttnDesc:
    """Descriptor from a query chunk [C][Hq][D] and a K pool [n_phys][Hkv][P][D]."""
    if grad_dtype is torch.float32 or grad_dtype is torch.bfloat16:
        desc = AttnDesc()
        if (_nb or _native()).make_desc(desc, q, k_pool, ctx_len, sm_scale, grad_dtype is torch.bfloat16) == 0:
            return desc
    C, Hq, D = q.shape
    n_phys, Hkv, P, D2 = k_pool.shape
    assert D == D2 and q.stride(2) == 1 and k_pool.stride(3) == 1
    return AttnDesc(Hq, Hkv, D, P, C, _dt(q.dtype), _dt(grad_dtype), float(sm_scale), int(ctx_len),
                    k_pool.stride(0), k_pool.stride(1), k_pool.stride(2), q.stride(0), q.stride(1), n_phys)


def _like(where: str, name: str, t: Optional[torch.Tensor], ref: torch.Tensor, dtype=None) -> None:
    """The descriptor carries ONE stride set for Q / O / dO / dQ and one for the K / V / dK / dV pools: every tensor of
    a family must have the shape and strides of the tensor the descriptor was made from (and the expected dtype)."""
    if t is None:
        return
    want = ref.dtype if dtype is None else dtype
    if tuple(t.shape) != tuple(ref.shape) or tuple(t.stride()) != tuple(ref.stride()) or t.dtype != want:
        raise OombError(ERR_INVALID_ARG, f"{where}: {name} must have shape {tuple(ref.shape)}, strides {tuple(ref.stride())} "
                                         f"and dtype {want} (got {tuple(t.shape)}, {tuple(t.stride())}, {t.dtype})")


def _check_family(where: str, desc: "AttnDesc", q, k_pool, rows=(), pools=(), grad_pools=(), lse=None) -> None:
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (desc.n_q_heads, desc.chunk_len) or
                            not lse.is_contiguous()):
        raise OombError(ERR_INVALID_ARG, f"{where}: lse must be a contiguous float32 [Hq][C] tensor")
    if (q.stride(0), q.stride(1)) != (desc.q_tok_stride, desc.q_head_stride) or _dt(q.dtype) != desc.dtype:
        raise OombError(ERR_INVALID_ARG, f"{where}: q does not match the descriptor's strides / dtype")
    if tuple(k_pool.stride()[:3]) != (desc.pool_page_stride, desc.pool_head_stride, desc.pool_tok_stride):
        raise OombError(ERR_INVALID_ARG, f"{where}: k_pool does not match the descriptor's strides")
    for name, t in rows:
        _like(where, name, t, q)
    for name, t in pools:
        _like(where, name, t, k_pool)
    gdt = torch.bfloat16 if desc.grad_dtype == BF16 else torch.float32
    for name, t in grad_pools:
        _like(where, name, t, k_pool, gdt)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(t: torch.Tensor):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def workspace_bytes(desc: AttnDesc, top_k: int, op: int) -> int:
    return int(lib().oomb_workspace_bytes(ctypes.byref(desc), int(top_k), int(op)))


def _workspace(desc, top_k, op, device):
    if _no_workspace(desc, top_k, op):
        raise OombError(ERR_INVALID_ARG, "oomb_workspace_bytes")
    return torch.empty(workspace_bytes(desc, top_k, op), dtype=torch.uint8, device=device)


def _failed(st: int, where: str, desc, top_k: int, op: int):
    """The error of a call that returned `st`."""
    if _no_workspace(desc, top_k, op):
        return OombError(ERR_INVALID_ARG, "oomb_workspace_bytes")
    return _refused(where) if st < 0 else OombError(st, where)


def page_score_topk(desc: AttnDesc, q, k_pool, page_table, top_k: int, sel_pages=None, sel_count=None,
                    scores_out=None, workspace=None):
    """oomb_page_score_topk.  Returns (sel_pages [Hkv][top_k + m] int32, sel_count [Hkv] int32)."""
    m = desc.chunk_len // desc.page_size
    if sel_pages is None:
        sel_pages = torch.empty((desc.n_kv_heads, top_k + m), dtype=torch.int32, device=q.device)
    if sel_count is None:
        sel_count = torch.empty((desc.n_kv_heads,), dtype=torch.int32, device=q.device)
    if workspace is None:
        workspace = _workspace(desc, top_k, OP_SCORE_TOPK, q.device)
    st = (_nb or _native()).score_topk(desc, q, k_pool, page_table, int(top_k), sel_pages, sel_count, scores_out, workspace)
    if st != OK:
        raise _failed(st, "oomb_page_score_topk", desc, top_k, OP_SCORE_TOPK)
    return sel_pages, sel_count


def page_score_topk_noalloc(desc: AttnDesc, q, k_pool, page_table, top_k: int, sel_pages, sel_count, scores_out=None):
    """oomb_page_score_topk_noalloc: every buffer is the caller's; nothing is allocated here either."""
    st = lib().oomb_page_score_topk_noalloc(ctypes.byref(desc), _p(q), _p(k_pool), _p(page_table), int(top_k),
                                            _p(sel_pages), _p(sel_count), _p(scores_out), _stream(q))
    if st != OK:
        raise OombError(st, "oomb_page_score_topk_noalloc")
    return sel_pages, sel_count


def _list_k(desc, sel_pages) -> int:
    """top_k of oomb_workspace_bytes for one list per KV head: the lists' row stride less the local pages, -1 without lists"""
    return -1 if sel_pages is None else int(sel_pages.stride(0)) - desc.chunk_len // desc.page_size


_SHORT_ROWS = -2   # of the native module: page lists whose last row ends with the memory before its stride does


def _whole_rows(sel_pages):
    """The same lists in memory of their own: the kernels read whole rows before they know how many entries are valid."""
    return sel_pages.clone(memory_format=torch.contiguous_format)


def paged_attn_fwd(desc: AttnDesc, q, k_pool, v_pool, page_table, sel_pages=None, sel_count=None, o=None,
                   lse=None, workspace=None):
    """oomb_paged_attn_fwd.  Returns (O [C][Hq][D], LSE [Hq][C] float32)."""
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((desc.n_q_heads, desc.chunk_len), dtype=torch.float32, device=q.device)
    if workspace is None:
        _check_family("oomb_paged_attn_fwd", desc, q, k_pool, rows=[("o", o)], pools=[("v_pool", v_pool)], lse=lse)
        workspace = _workspace(desc, _list_k(desc, sel_pages), OP_ATTN_FWD, q.device)
    st = (_nb or _native()).attn_fwd(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, workspace)
    if st == _SHORT_ROWS:
        st = _native().attn_fwd(desc, q, k_pool, v_pool, page_table, _whole_rows(sel_pages), sel_count, o, lse, workspace)
    if st != OK:
        _check_family("oomb_paged_attn_fwd", desc, q, k_pool, rows=[("o", o)], pools=[("v_pool", v_pool)], lse=lse)
        raise _failed(st, "oomb_paged_attn_fwd", desc, _list_k(desc, sel_pages), OP_ATTN_FWD)
    return o, lse


def paged_attn_bwd(desc: AttnDesc, q, k_pool, v_pool, page_table, o, lse, d_o, dk_pool, dv_pool,
                   sel_pages=None, sel_count=None, d_q=None, workspace=None):
    """oomb_paged_attn_bwd.  Returns dQ; dk_pool / dv_pool are accumulated in place."""
    if d_q is None:
        d_q = torch.empty_like(q)
    def check():
        _check_family("oomb_paged_attn_bwd", desc, q, k_pool, rows=[("o", o), ("d_o", d_o), ("d_q", d_q)],
                      pools=[("v_pool", v_pool)], grad_pools=[("dk_pool", dk_pool), ("dv_pool", dv_pool)], lse=lse)
    if workspace is None:
        check()
        workspace = _workspace(desc, _list_k(desc, sel_pages), OP_ATTN_BWD, q.device)
    st = (_nb or _native()).attn_bwd(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, d_o, d_q, dk_pool, dv_pool, workspace)
    if st == _SHORT_ROWS:
        st = _native().attn_bwd(desc, q, k_pool, v_pool, page_table, _whole_rows(sel_pages), sel_count, o, lse, d_o, d_q, dk_pool, dv_pool, workspace)
    if st != OK:
        check()
        raise _failed(st, "oomb_paged_attn_bwd", desc, _list_k(desc, sel_pages), OP_ATTN_BWD)
    return d_q


def page_vote_topk(desc: AttnDesc, q, kbar_cache, top_k: int, sel_pages=None, sel_count=None, votes_out=None,
                   workspace=None):
    """oomb_page_vote_topk.  Returns (sel_pages [Hkv][m][top_k + m] int32, sel_count [Hkv][m] int32)."""
    m = desc.chunk_len // desc.page_size
    if sel_pages is None:
        sel_pages = torch.empty((desc.n_kv_heads, m, top_k + m), dtype=torch.int32, device=q.device)
    if sel_count is None:
        sel_count = torch.empty((desc.n_kv_heads, m), dtype=torch.int32, device=q.device)
    if workspace is None:
        workspace = _workspace(desc, top_k, OP_VOTE_TOPK, q.device)
    st = (_nb or _native()).vote_topk(desc, q, kbar_cache, top_k, sel_pages, sel_count, votes_out, workspace)
    if st != OK:
        raise _failed(st, "oomb_page_vote_topk", desc, top_k, OP_VOTE_TOPK)
    return sel_pages, sel_count


def _stream_of(stream, t):
    return ctypes.c_void_p(stream.cuda_stream) if stream is not None else _stream(t)


def check_inputs(desc: AttnDesc, page_table, sel_pages=None, sel_count=None) -> int:
    """oomb_check_inputs: the violation bits (0 = the documented preconditions hold).  Synchronises."""
    dev = page_table.device
    out = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = torch.empty(max(workspace_bytes(desc, 0, OP_CHECK_INPUTS), 256), dtype=torch.uint8, device=dev)
    stride = lists = 0
    if sel_pages is not None:
        assert sel_pages.dim() in (2, 3) and sel_pages.is_contiguous() and sel_count.is_contiguous()
        stride = int(sel_pages.shape[-1])
        lists = 1 if sel_pages.dim() == 2 else int(sel_pages.shape[1])
    st = lib().oomb_check_inputs(ctypes.byref(desc), _p(page_table), _p(sel_pages), _p(sel_count), stride, lists, _p(out),
                                 _p(ws), ws.numel(), _stream(page_table))
    if st != OK:
        raise OombError(st, "oomb_check_inputs")
    return int(out.item())


class OffloadPlan:
    """Device arrays written by oomb_offload_plan (see include/oomb.h)."""

    def __init__(self, desc, capacity, device):
        n = desc.ctx_len // desc.page_size
        self.capacity = int(capacity)
        self.stage_table = torch.empty(n, dtype=torch.int32, device=device)
        self.slot_pages = torch.empty(self.capacity, dtype=torch.int32, device=device)
        self.head_mask = torch.empty(n, dtype=torch.int32, device=device)   # bit patterns of uint32
        self.n_slots = torch.empty(2, dtype=torch.int32, device=device)   # [slots in use, pages held]

    def overflowed(self) -> bool:
        """True iff the lists held more pages than the staging pools have slots (synchronises)."""
        return int(self.n_slots[1].item()) > self.capacity


def offload_capacity(desc: AttnDesc, sel_pages) -> int:
    """Slots that always suffice for lists of this shape: min(n, Hkv * lists per head * row stride)."""
    n = desc.ctx_len // desc.page_size
    return min(n, sel_pages.numel())


def offload_plan(desc: AttnDesc, sel_pages, sel_count, plan: "OffloadPlan" = None, stream=None) -> "OffloadPlan":
    """oomb_offload_plan for lists [Hkv][stride] or [Hkv][m][stride].  plan.stage_table is the page table to give
    the attention calls that run on the staging pools; plan.capacity must be the staging pools' page count."""
    assert sel_pages.dim() in (2, 3) and sel_pages.is_contiguous() and sel_count.is_contiguous()
    lists_per_head = 1 if sel_pages.dim() == 2 else int(sel_pages.shape[1])
    if plan is None:
        plan = OffloadPlan(desc, offload_capacity(desc, sel_pages), sel_pages.device)
    st = lib().oomb_offload_plan(ctypes.byref(desc), _p(sel_pages), _p(sel_count), int(sel_pages.shape[-1]), lists_per_head,
                                 plan.capacity, _p(plan.stage_table), _p(plan.slot_pages), _p(plan.head_mask), _p(plan.n_slots),
                                 _stream_of(stream, sel_pages))
    if st != OK:
        raise OombError(st, "oomb_offload_plan")
    return plan


def offload_fetch(desc: AttnDesc, host_k_pool, host_v_pool, page_table, plan: "OffloadPlan", stage_k, stage_v,
                  stage_dk=None, stage_dv=None, stream=None) -> None:
    """oomb_offload_fetch: host_*_pool are pinned host tensors (or device tensors) with the pools' layout; the
    staging pools hold stage_k.shape[0] pages."""
    if int(stage_k.shape[0]) != plan.capacity:
        raise OombError(ERR_INVALID_ARG, "oomb_offload_fetch (staging pool size differs from the plan's capacity)")
    _like("oomb_offload_fetch", "host_v_pool", host_v_pool, host_k_pool)
    _like("oomb_offload_fetch", "stage_v", stage_v, stage_k)
    gdt = torch.bfloat16 if desc.grad_dtype == BF16 else torch.float32
    _like("oomb_offload_fetch", "stage_dk", stage_dk, stage_k, gdt)
    _like("oomb_offload_fetch", "stage_dv", stage_dv, stage_k, gdt)
    if tuple(host_k_pool.stride()[1:]) != tuple(stage_k.stride()[1:]) or host_k_pool.dtype != stage_k.dtype or \
            tuple(stage_k.stride()[:3]) != (desc.pool_page_stride, desc.pool_head_stride, desc.pool_tok_stride):
        raise OombError(ERR_INVALID_ARG, "oomb_offload_fetch: host and staging pools must share the descriptor's strides and dtype")
    st = lib().oomb_offload_fetch(ctypes.byref(desc), _p(host_k_pool), _p(host_v_pool), _p(page_table), _p(plan.slot_pages),
                                  _p(plan.head_mask), _p(plan.n_slots), int(stage_k.shape[0]), _p(stage_k), _p(stage_v),
                                  _p(stage_dk), _p(stage_dv), _stream_of(stream, stage_k))
    if st != OK:
        raise OombError(st, "oomb_offload_fetch")


def offload_writeback(desc: AttnDesc, stage_dk, stage_dv, host_dk_pool, host_dv_pool, page_table, plan: "OffloadPlan",
                      stream=None) -> None:
    """oomb_offload_writeback: host pools += the staged gradient tiles of the held (page, KV head) pairs."""
    if int(stage_dk.shape[0]) != plan.capacity:
        raise OombError(ERR_INVALID_ARG, "oomb_offload_writeback (staging pool size differs from the plan's capacity)")
    gdt = torch.bfloat16 if desc.grad_dtype == BF16 else torch.float32
    _like("oomb_offload_writeback", "stage_dv", stage_dv, stage_dk, gdt)
    _like("oomb_offload_writeback", "host_dv_pool", host_dv_pool, host_dk_pool, gdt)
    if tuple(host_dk_pool.stride()[1:]) != tuple(stage_dk.stride()[1:]) or stage_dk.dtype != gdt or \
            tuple(stage_dk.stride()[:3]) != (desc.pool_page_stride, desc.pool_head_stride, desc.pool_tok_stride):
        raise OombError(ERR_INVALID_ARG, "oomb_offload_writeback: host and staging pools must share the descriptor's strides and dtype")
    st = lib().oomb_offload_writeback(ctypes.byref(desc), _p(stage_dk), _p(stage_dv), _p(host_dk_pool), _p(host_dv_pool),
                                      _p(page_table), _p(plan.slot_pages), _p(plan.head_mask), _p(plan.n_slots),
                                      int(stage_dk.shape[0]), _stream_of(stream, stage_dk))
    if st != OK:
        raise OombError(st, "oomb_offload_writeback")


def _qp_lists(desc, sel_pages, sel_count):
    m = desc.chunk_len // desc.page_size
    assert sel_pages.dim() == 3 and sel_pages.shape[:2] == (desc.n_kv_heads, m) and sel_pages.is_contiguous()
    assert sel_count.shape == (desc.n_kv_heads, m) and sel_count.is_contiguous()
    return int(sel_pages.shape[2]), m


def paged_attn_fwd_qp(desc: AttnDesc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o=None, lse=None,
                      workspace=None):
    """oomb_paged_attn_fwd_qp: one list per (KV head, query page), sel_pages [Hkv][m][stride] int32,
    sel_count [Hkv][m].  Returns (O, LSE)."""
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((desc.n_q_heads, desc.chunk_len), dtype=torch.float32, device=q.device)
    def check():
        _check_family("oomb_paged_attn_fwd_qp", desc, q, k_pool, rows=[("o", o)], pools=[("v_pool", v_pool)], lse=lse)
        stride, m = _qp_lists(desc, sel_pages, sel_count)
        return stride - m
    if workspace is None:
        workspace = _workspace(desc, check(), OP_ATTN_FWD_QP, q.device)
    st = (_nb or _native()).attn_fwd_qp(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, workspace)
    if st != OK:
        raise _failed(st, "oomb_paged_attn_fwd_qp", desc, check(), OP_ATTN_FWD_QP)
    return o, lse


def paged_attn_bwd_qp(desc: AttnDesc, q, k_pool, v_pool, page_table, o, lse, d_o, dk_pool, dv_pool, sel_pages,
                      sel_count, d_q=None, workspace=None):
    """oomb_paged_attn_bwd_qp.  Returns dQ; dk_pool / dv_pool are accumulated in place."""
    if d_q is None:
        d_q = torch.empty_like(q)
    def check():
        _check_family("oomb_paged_attn_bwd_qp", desc, q, k_pool, rows=[("o", o), ("d_o", d_o), ("d_q", d_q)],
                      pools=[("v_pool", v_pool)], grad_pools=[("dk_pool", dk_pool), ("dv_pool", dv_pool)], lse=lse)
        stride, m = _qp_lists(desc, sel_pages, sel_count)
        return stride - m
    if workspace is None:
        workspace = _workspace(desc, check(), OP_ATTN_BWD_QP, q.device)
    st = (_nb or _native()).attn_bwd_qp(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, d_o, d_q, dk_pool, dv_pool, workspace)
    if st != OK:
        raise _failed(st, "oomb_paged_attn_bwd_qp", desc, check(), OP_ATTN_BWD_QP)
    return d_q


def profile_enable(on) -> None:
    """oomb_profile_enable: 1 / True brackets every kernel launch with HIP events on the launch stream,
    2 only the large kernels, 0 / False none."""
    lib().oomb_profile_enable(int(on))


def profile_reset() -> None:
    lib().oomb_profile_reset()


def profile_read() -> dict:
    """oomb_profile_read for every entry: {kernel name: (total_ms, launches)}."""
    out = {}
    for idx in range(lib().oomb_profile_count()):
        name = ctypes.create_string_buffer(64)
        ms = ctypes.c_double()
        n = ctypes.c_int64()
        st = lib().oomb_profile_read(idx, name, 64, ctypes.byref(ms), ctypes.byref(n))
        if st != OK:
            raise OombError(st, "oomb_profile_read")
        out[name.value.decode()] = (ms.value, n.value)
    return out


def calibrate(which: int, buf) -> float:
    """oomb_calibrate: measured ceiling of the device (0: bf16 MFMA TFLOP/s on constant operands, 2: on random
    operands, 1: copy GB/s, read + write)."""
    out = ctypes.c_double()
    st = lib().oomb_calibrate(int(which), _p(buf), buf.numel() * buf.element_size(), ctypes.byref(out), _stream(buf))
    if st != OK:
        raise OombError(st, "oomb_calibrate")
    return out.value


def kv_append(desc: AttnDesc, k_chunk, v_chunk, page_table, k_pool, v_pool, kbar_cache=None) -> None:
    """oomb_kv_append: the chunk's K / V [C][Hkv][D] into its local pages (+ their means into kbar_cache)."""
    st = (_nb or _native()).kv_append(desc, k_chunk, v_chunk, page_table, k_pool, v_pool, kbar_cache)
    if st == OK:
        return
    if not (k_chunk.is_contiguous() and v_chunk.is_contiguous()) or k_chunk.shape != v_chunk.shape or \
            k_chunk.dtype != k_pool.dtype or v_chunk.dtype != k_pool.dtype:
        raise OombError(ERR_INVALID_ARG, "oomb_kv_append: k_chunk / v_chunk must be contiguous [C][Hkv][D] of the pools' dtype")
    _like("oomb_kv_append", "v_pool", v_pool, k_pool)
    raise _refused("oomb_kv_append") if st < 0 else OombError(st, "oomb_kv_append")


class PagePool:
    """Free list of the physical pages that the K / V / dK / dV pools share (oomb_page_pool_*): host-side state
    (a stack of page ids and its fill level) held here, every operation done by the library."""

    def __init__(self, num_phys_pages: int):
        self.num_phys_pages = int(num_phys_pages)
        self._stack = (ctypes.c_int32 * max(self.num_phys_pages, 1))()
        self._n_free = ctypes.c_int64(0)
        st = lib().oomb_page_pool_reset(self.num_phys_pages, self._stack, ctypes.byref(self._n_free))
        if st != OK:
            raise OombError(st, "oomb_page_pool_reset")

    @property
    def n_free(self) -> int:
        return int(self._n_free.value)

    def alloc(self, count: int) -> list:
        out = (ctypes.c_int32 * max(int(count), 1))()
        st = lib().oomb_page_pool_alloc(self._stack, ctypes.byref(self._n_free), int(count), out)
        if st != OK:
            raise OombError(st, "oomb_page_pool_alloc")
        return list(out[: int(count)])

    def release(self, pages) -> None:
        pages = [int(x) for x in pages]
        arr = (ctypes.c_int32 * max(len(pages), 1))(*pages)
        st = lib().oomb_page_pool_release(self.num_phys_pages, self._stack, ctypes.byref(self._n_free), arr, len(pages))
        if st != OK:
            raise OombError(st, "oomb_page_pool_release")


def page_means(desc: AttnDesc, k_pool, page_table, first_page: int, n_pages: int, kbar_cache) -> None:
    """oomb_page_means: means of logical pages [first_page, first_page + n_pages) into kbar_cache."""
    st = lib().oomb_page_means(ctypes.byref(desc), _p(k_pool), _p(page_table), int(first_page), int(n_pages),
                               _p(kbar_cache), _stream(k_pool))
    if st != OK:
        raise OombError(st, "oomb_page_means")


def page_score_topk_cached(desc: AttnDesc, q, kbar_cache, top_k: int, sel_pages=None, sel_count=None,
                           scores_out=None, workspace=None):
    """oomb_page_score_topk_cached.  Returns (sel_pages [Hkv][top_k + m] int32, sel_count [Hkv] int32)."""
    m = desc.chunk_len // desc.page_size
    if sel_pages is None:
        sel_pages = torch.empty((desc.n_kv_heads, top_k + m), dtype=torch.int32, device=q.device)
    if sel_count is None:
        sel_count = torch.empty((desc.n_kv_heads,), dtype=torch.int32, device=q.device)
    if workspace is None:
        workspace = _workspace(desc, top_k, OP_SCORE_TOPK, q.device)
    st = (_nb or _native()).score_topk_cached(desc, q, kbar_cache, int(top_k), sel_pages, sel_count, scores_out, workspace)
    if st != OK:
        raise _failed(st, "oomb_page_score_topk_cached", desc, top_k, OP_SCORE_TOPK)
    return sel_pages, sel_count


def local_page_list(desc: AttnDesc, window_pages: int, device, sel_pages=None, sel_count=None):
    """oomb_local_page_list.  Returns (sel_pages [Hkv][window_pages + m] int32, sel_count [Hkv] int32)."""
    m = desc.chunk_len // desc.page_size
    if sel_pages is None:
        sel_pages = torch.empty((desc.n_kv_heads, window_pages + m), dtype=torch.int32, device=device)
    if sel_count is None:
        sel_count = torch.empty((desc.n_kv_heads,), dtype=torch.int32, device=device)
    st = (_nb or _native()).local_page_list(desc, int(window_pages), sel_pages, sel_count)
    if st != OK:
        raise _refused("oomb_local_page_list") if st < 0 else OombError(st, "oomb_local_page_list")
    return sel_pages, sel_count


# ---- packed rows of any number of sequences: rotation and append, their backward, a cache held in 4 bits (include/oomb.h) ----
# (row tensors that a call makes itself are zero where it writes nothing: rows of no sequence, or in front of its first token)

class Rope:
    """Tables of a position rotation: cos, sin [positions][rot_dim / 2] float32; pairs in halves, or neighbours."""
    __slots__ = ("cos", "sin", "interleaved")

    def __init__(self, cos, sin, interleaved: bool = False):
        self.cos, self.sin, self.interleaved = cos, sin, bool(interleaved)


def rope_tables(n_pos: int, rot_dim: int, theta: float = 10000.0, interleaved: bool = False, device="cuda") -> Rope:
    """Rope with the angles p * theta^(-2 i / rot_dim), taken in 64 bits (far positions), held in 32."""
    half = rot_dim // 2
    freq = float(theta) ** (-torch.arange(half, dtype=torch.float64) / half)
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * freq
    return Rope(angle.cos().float().to(device), angle.sin().float().to(device), interleaved)


def kvq_tile_bytes(page_size: int, head_dim: int) -> int:
    """Bytes of one page of one KV head in a pool of 4-bit codes."""
    return page_size * (head_dim // 2 + head_dim // 32)


def kvq_pool(n_phys: int, n_kv_heads: int, page_size: int, head_dim: int, device="cuda") -> torch.Tensor:
    """A pool of 4-bit codes, uint8 [n_phys][Hkv][tile]."""
    return torch.zeros((n_phys, n_kv_heads, kvq_tile_bytes(page_size, head_dim)), dtype=torch.uint8, device=device)


def make_rows_desc(q: torch.Tensor, pool: torch.Tensor, page_tables: torch.Tensor, max_len: int, sm_scale: float = 1.0,
                   max_rows: Optional[int] = None) -> RowsDesc:
    """Descriptor from packed rows [n_rows][Hq][D], a pool ([n_phys][Hkv][P][D], or a kvq_pool) and page tables ([n_seqs][pages], or
    [pages] of one sequence).  max_rows: most rows of one sequence (default: all rows)."""
    desc = RowsDesc()
    if (_nb or _native()).make_rows_desc(desc, q, pool, page_tables, max_len, sm_scale, max_rows or 0) != 0:
        raise OombError(ERR_INVALID_ARG, "make_rows_desc: q must be [n_rows][Hq][D] float32 or bfloat16, pool [n_phys][Hkv][P][D] or a kvq_pool "
                                         "of that head dim, page_tables [n_seqs][pages] or [pages]")
    return desc


def means_desc(q: torch.Tensor, n_kv_heads: int, page_size: int, ctx_len: int, sm_scale: float) -> AttnDesc:
    """AttnDesc for the calls that pick pages from cached means (page_score_topk_cached, page_vote_topk, local_page_list) where
    there is no K pool of q's type to make it from: a chunk [C][Hq][D] of whole pages over a cache held in 4 bits."""
    C, Hq, D = q.shape
    return AttnDesc(Hq, n_kv_heads, D, page_size, C, _dt(q.dtype), F32, float(sm_scale), int(ctx_len), n_kv_heads * page_size * D, page_size * D, D,
                    q.stride(0), q.stride(1), ctx_len // page_size)


def _rows_refused(where: str, desc: RowsDesc, rows, pools, page_tables, seq_lens, row_starts, rope=None, kbar_cache=None, others=()):
    """The error of a call whose tensors the native module did not take: which of them does not fit the descriptor."""
    def bad(what):
        return OombError(ERR_INVALID_ARG, f"{where}: {what}")

    dt = torch.bfloat16 if desc.dtype == BF16 else torch.float32
    kvq_shape = (desc.num_phys_pages, desc.n_kv_heads, kvq_tile_bytes(desc.page_size, desc.head_dim))
    pages = -(-desc.max_len // max(desc.page_size, 1))
    tensors = []
    for name, t, heads in rows:
        want = (desc.n_rows, heads, desc.head_dim)
        if not isinstance(t, torch.Tensor) or tuple(t.shape) != want or t.dtype != dt or t.stride(2) != 1:
            return bad(f"{name} must be {list(want)}, {dt}, its last dim contiguous")
        tensors.append((name, t))
    for name, t, kind in pools:
        want = kvq_shape if kind is torch.uint8 else (desc.num_phys_pages, desc.n_kv_heads, desc.page_size, desc.head_dim)
        strides = (desc.pool_page_stride, desc.pool_head_stride) + (() if kind is torch.uint8 else (desc.pool_tok_stride,)) + (1,)
        if not isinstance(t, torch.Tensor) or tuple(t.shape) != want or tuple(t.stride()) != strides or t.dtype != kind:
            return bad(f"{name} must be {list(want)}, {kind}, with the strides {list(strides)} of the descriptor's pool")
        tensors.append((name, t))
    t = page_tables
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or (t.dim() == 1 and desc.n_seqs != 1) or t.dim() not in (1, 2) or \
            (t.dim() == 2 and (t.shape[0] != desc.n_seqs or (desc.n_seqs > 1 and t.stride(0) != desc.table_stride))) or t.shape[-1] < pages or \
            (t.shape[-1] > 1 and t.stride(-1) != 1):
        return bad(f"page_tables must be int32 [{desc.n_seqs}][>= {pages}] with the descriptor's row stride")
    tensors.append(("page_tables", t))
    for name, t, n in (("seq_lens", seq_lens, desc.n_seqs), ("row_starts", row_starts, desc.n_seqs + 1)):
        if t is not None and (not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or tuple(t.shape) != (n,) or not t.is_contiguous()):
            return bad(f"{name} must be contiguous int32 [{n}]")
        tensors.append((name, t))
    if rope is not None:
        for name in ("cos", "sin"):
            t = getattr(rope, name)
            if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.shape != rope.cos.shape:
                return bad("rope.cos and rope.sin must be contiguous float32 [positions][rot_dim / 2]")
            tensors.append((name, t))
    if kbar_cache is not None:
        t = kbar_cache
        if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or not t.is_contiguous() or t.dim() not in (3, 4) or \
                tuple(t.shape[-2:]) != (desc.n_kv_heads, desc.head_dim) or (t.dim() == 3 and desc.n_seqs != 1) or \
                (t.dim() == 4 and (t.shape[0] != desc.n_seqs or (desc.n_seqs > 1 and t.shape[1] != desc.table_stride))) or t.shape[-3] < pages:
            return bad("kbar_cache must be contiguous float32 [n_seqs][table stride][Hkv][D] ([pages][Hkv][D] for one sequence)")
        tensors.append(("kbar_cache", t))
    tensors += list(others)
    devices = {t.device for _, t in tensors if t is not None}
    if len(devices) > 1 or any(x.type != "cuda" for x in devices):
        return bad(f"the tensors must lie on one GPU (got {sorted(str(x) for x in devices)})")
    return _refused(where)


def _new_rows(desc, heads, device, every_row: bool):
    """A new row tensor for a call that writes every row, or leaves some alone: those start at zero."""
    make = torch.empty if every_row else torch.zeros
    return make((desc.n_rows, heads, desc.head_dim), dtype=torch.bfloat16 if desc.dtype == BF16 else torch.float32, device=device)


def _all_exist(desc, seq_lens, row_starts) -> bool:
    """Whether every row is sure to be a token of a sequence.  With lengths on the device, a sequence may be shorter than its rows."""
    return row_starts is None and seq_lens is None and desc.n_rows <= desc.n_seqs * desc.max_len


def _rope(rope):
    return (None, None, False) if rope is None else (rope.cos, rope.sin, bool(rope.interleaved))


def _append_rope(where, native, pool_dtype, desc, k, v, page_tables, k_pool, v_pool, q, q_out, rope, kbar_cache, seq_lens, row_starts):
    if q is not None and q_out is None:
        q_out = _new_rows(desc, desc.n_q_heads, q.device, _all_exist(desc, seq_lens, row_starts))
    st = native(desc, *_rope(rope), q, q_out, k, v, page_tables, seq_lens, row_starts, k_pool, v_pool, kbar_cache)
    if st < 0:
        rows = [("k", k, desc.n_kv_heads), ("v", v, desc.n_kv_heads)]
        if q is not None or q_out is not None:
            rows += [("q", q, desc.n_q_heads), ("q_out", q_out, desc.n_q_heads)]
        raise _rows_refused(where, desc, rows, [("k_pool", k_pool, pool_dtype), ("v_pool", v_pool, pool_dtype)], page_tables, seq_lens, row_starts, rope,
                            kbar_cache)
    if st != OK:
        raise OombError(st, where)
    return q_out


def kv_append_rope(desc: RowsDesc, k, v, page_tables, k_pool, v_pool, q=None, q_out=None, rope: Optional[Rope] = None, kbar_cache=None, seq_lens=None,
                   row_starts=None):
    """oomb_kv_append_rope: the rows' keys, rotated, and values into their pages (+ the means of the pages they fill into kbar_cache).
    Returns q rotated (q_out, a new tensor unless given, zero where rows do not exist; None without q)."""
    return _append_rope("oomb_kv_append_rope", (_nb or _native()).kv_append_rope, torch.bfloat16 if desc.dtype == BF16 else torch.float32, desc, k, v,
                        page_tables, k_pool, v_pool, q, q_out, rope, kbar_cache, seq_lens, row_starts)


def kvq_append_rope(desc: RowsDesc, k, v, page_tables, k_pool, v_pool, q=None, q_out=None, rope: Optional[Rope] = None, kbar_cache=None, seq_lens=None,
                    row_starts=None):
    """oomb_kvq_append_rope: kv_append_rope into pools of 4-bit codes (kvq_pool)."""
    return _append_rope("oomb_kvq_append_rope", (_nb or _native()).kvq_append_rope, torch.uint8, desc, k, v, page_tables, k_pool, v_pool, q, q_out, rope,
                        kbar_cache, seq_lens, row_starts)


def kv_append_rope_bwd(desc: RowsDesc, dk_pool, dv_pool, page_tables, d_q=None, rope: Optional[Rope] = None, d_q_out=None, d_k=None, d_v=None,
                       seq_lens=None, row_starts=None):
    """oomb_kv_append_rope_bwd: the gradients with respect to the rows that kv_append_rope took, from d_q (of its q_out) and the gradient pools
    (float32 or bfloat16; desc made with one of them as the pool).  Returns (d_q_out, d_k, d_v), d_q_out None without d_q."""
    def new(heads):
        return _new_rows(desc, heads, dk_pool.device, _all_exist(desc, seq_lens, row_starts))
    if d_q is not None and d_q_out is None:
        d_q_out = new(desc.n_q_heads)
    if d_k is None:
        d_k = new(desc.n_kv_heads)
    if d_v is None:
        d_v = new(desc.n_kv_heads)
    st = (_nb or _native()).kv_append_rope_bwd(desc, *_rope(rope), d_q, d_q_out, d_k, d_v, page_tables, seq_lens, row_starts, dk_pool, dv_pool)
    if st < 0:
        rows = [("d_k", d_k, desc.n_kv_heads), ("d_v", d_v, desc.n_kv_heads)]
        if d_q is not None or d_q_out is not None:
            rows += [("d_q", d_q, desc.n_q_heads), ("d_q_out", d_q_out, desc.n_q_heads)]
        gdt = dk_pool.dtype if dk_pool.dtype == torch.bfloat16 else torch.float32
        raise _rows_refused("oomb_kv_append_rope_bwd", desc, rows, [("dk_pool", dk_pool, gdt), ("dv_pool", dv_pool, gdt)], page_tables, seq_lens, row_starts, rope)
    if st != OK:
        raise OombError(st, "oomb_kv_append_rope_bwd")
    return d_q_out, d_k, d_v


def kvq_read(desc: RowsDesc, k_pool, v_pool, page_tables, k_out=None, v_out=None, seq_lens=None, row_starts=None):
    """oomb_kvq_read: the rows' values as a cache of 4-bit codes holds them.  Returns (k [n_rows][Hkv][D], v)."""
    k_out, v_out = (_new_rows(desc, desc.n_kv_heads, k_pool.device, _all_exist(desc, seq_lens, row_starts)) if t is None else t for t in (k_out, v_out))
    st = (_nb or _native()).kvq_read(desc, page_tables, seq_lens, row_starts, k_pool, v_pool, k_out, v_out)
    if st < 0:
        raise _rows_refused("oomb_kvq_read", desc, [("k_out", k_out, desc.n_kv_heads), ("v_out", v_out, desc.n_kv_heads)],
                            [("k_pool", k_pool, torch.uint8), ("v_pool", v_pool, torch.uint8)], page_tables, seq_lens, row_starts)
    if st != OK:
        raise OombError(st, "oomb_kvq_read")
    return k_out, v_out


def kvq_workspace_bytes(desc: RowsDesc, sel_stride: int = -1) -> int:
    """oomb_kvq_workspace_bytes: what paged_attn_fwd_kvq needs with lists of this row stride (-1: every page); may be 0."""
    return int(lib().oomb_kvq_workspace_bytes(ctypes.byref(desc), int(sel_stride)))


def rows_workspace_bytes(desc: RowsDesc, sel_stride: int = -1) -> int:
    """oomb_rows_workspace_bytes: what paged_attn_fwd_rows needs with lists of this row stride (-1: every page); may be 0."""
    return int(lib().oomb_rows_workspace_bytes(ctypes.byref(desc), int(sel_stride)))


def _attn_fwd_packed(where, native, workspace_bytes, pool_dtype, desc, q, k_pool, v_pool, page_tables, sel_pages, sel_count, o, lse, workspace, seq_lens,
                     row_starts):
    if o is None:
        o = _new_rows(desc, desc.n_q_heads, q.device, row_starts is None)   # (a row that does not exist gets zeros from the call)
    if lse is None:
        lse = (torch.empty if row_starts is None else torch.zeros)((desc.n_q_heads, desc.n_rows), dtype=torch.float32, device=q.device)
    if workspace is None:
        need = workspace_bytes(desc, -1 if sel_pages is None else int(sel_pages.shape[-1]))
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    st = native(desc, q, k_pool, v_pool, page_tables, seq_lens, row_starts, sel_pages, sel_count, o, lse, workspace)
    if st < 0:
        lists = desc.n_seqs * desc.n_kv_heads
        if lse.dtype != torch.float32 or tuple(lse.shape) != (desc.n_q_heads, desc.n_rows) or not lse.is_contiguous():
            raise OombError(ERR_INVALID_ARG, f"{where}: lse must be contiguous float32 [{desc.n_q_heads}][{desc.n_rows}]")
        if sel_pages is not None and (sel_count is None or sel_pages.dtype != torch.int32 or sel_count.dtype != torch.int32 or sel_pages.dim() < 2 or
                                      not sel_pages.is_contiguous() or not sel_count.is_contiguous() or sel_count.numel() != lists or
                                      sel_pages.numel() != lists * sel_pages.shape[-1]):
            raise OombError(ERR_INVALID_ARG, f"{where}: sel_pages must be contiguous int32 [n_seqs][Hkv][stride], sel_count [n_seqs][Hkv]")
        raise _rows_refused(where, desc, [("q", q, desc.n_q_heads), ("o", o, desc.n_q_heads)],
                            [("k_pool", k_pool, pool_dtype), ("v_pool", v_pool, pool_dtype)], page_tables, seq_lens, row_starts,
                            others=[("sel_pages", sel_pages), ("sel_count", sel_count), ("lse", lse), ("workspace", workspace)])
    if st != OK:
        raise OombError(st, where)
    return o, lse


def paged_attn_fwd_kvq(desc: RowsDesc, q, k_pool, v_pool, page_tables, sel_pages=None, sel_count=None, o=None, lse=None, workspace=None, seq_lens=None,
                       row_starts=None):
    """oomb_paged_attn_fwd_kvq: attention of the rows over a cache of 4-bit codes, every page or lists [n_seqs][Hkv][stride] ([Hkv][stride] for
    one sequence).  Returns (O [n_rows][Hq][D], LSE [Hq][n_rows] float32)."""
    return _attn_fwd_packed("oomb_paged_attn_fwd_kvq", (_nb or _native()).attn_fwd_kvq, kvq_workspace_bytes, torch.uint8, desc, q, k_pool, v_pool, page_tables,
                            sel_pages, sel_count, o, lse, workspace, seq_lens, row_starts)


def paged_attn_fwd_rows(desc: RowsDesc, q, k_pool, v_pool, page_tables, sel_pages=None, sel_count=None, o=None, lse=None, workspace=None, seq_lens=None,
                        row_starts=None):
    """oomb_paged_attn_fwd_rows: paged_attn_fwd_kvq over pools [n_phys][Hkv][P][D] of the rows' type."""
    return _attn_fwd_packed("oomb_paged_attn_fwd_rows", (_nb or _native()).attn_fwd_rows, rows_workspace_bytes,
                            torch.bfloat16 if desc.dtype == BF16 else torch.float32, desc, q, k_pool, v_pool, page_tables, sel_pages, sel_count, o, lse,
                            workspace, seq_lens, row_starts)


# ---- generation with several hypotheses a text: the steps between two passes of attention (include/oomb.h) ----

FORK_NONE, FORK_BEGINS = -1, -2   # parents of a sequence that holds nothing, and of one that begins


class PageFork:
    """What page_fork leaves: tables [n_out][cols], lens [n_out], refs [n_phys], copies [n_out][3] (for page_copy), status [2] (pages taken, pages missing)."""
    __slots__ = ("tables", "lens", "refs", "copies", "status")

    def __init__(self, tables, lens, refs, copies, status):
        self.tables, self.lens, self.refs, self.copies, self.status = tables, lens, refs, copies, status


class PageCompact:
    """What page_compact leaves: tables, refs, moves [n_phys / 2][3] (for page_copy, status[1:] of them), page_map [n_phys], status [2] (used pages, moves)."""
    __slots__ = ("tables", "refs", "moves", "page_map", "status")

    def __init__(self, tables, refs, moves, page_map, status):
        self.tables, self.refs, self.moves, self.page_map, self.status = tables, refs, moves, page_map, status


def _gen_refused(where: str, ints=(), floats=(), others=()):
    """The error of a call whose tensors the native module did not take.  ints, floats: (name, tensor, shape; None in it: any size)."""
    tensors = list(others)
    for dt, group in ((torch.int32, ints), (torch.float32, floats)):
        for name, t, shape in group:
            if t is None:
                continue
            if not isinstance(t, torch.Tensor) or t.dtype != dt or t.dim() != len(shape) or any(n is not None and t.shape[i] != n for i, n in enumerate(shape)) or \
                    (t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1):
                return OombError(ERR_INVALID_ARG, f"{where}: {name} must be {dt} {['any' if n is None else n for n in shape]}, its last dim contiguous")
            tensors.append((name, t))
    devices = {t.device for _, t in tensors if isinstance(t, torch.Tensor)}
    if len(devices) > 1 or any(x.type != "cuda" for x in devices):
        return OombError(ERR_INVALID_ARG, f"{where}: the tensors must lie on one GPU (got {sorted(str(x) for x in devices)})")
    return _refused(where)


def _n(t, dim=0):
    return int(t.shape[dim]) if isinstance(t, torch.Tensor) and t.dim() > dim else None


def _workspace_of(need: int, device):
    return torch.empty(max(need, 16), dtype=torch.uint8, device=device)


def page_fork_workspace_bytes(n_seqs: int, n_out: int, n_phys: int) -> int:
    """oomb_page_fork_workspace_bytes."""
    return int(lib().oomb_page_fork_workspace_bytes(int(n_seqs), int(n_out), int(n_phys)))


def page_fork(page_tables, seq_lens, parents, refs, page_size: int, grow=None, tables_out=None, lens_out=None, refs_out=None, copies=None, status=None,
              workspace=None) -> PageFork:
    """oomb_page_fork: the sequences of the next step, one per entry of parents (a sequence, FORK_BEGINS or FORK_NONE), each with room for
    grow more tokens.  refs is updated in place unless refs_out is given.  page_copy(pools, result.copies) then copies the partly filled pages.
    What the caller keeps by sequence (page means, texts, who has ended) it gathers by parents itself."""
    for name, t, dims in (("page_tables", page_tables, 2), ("seq_lens", seq_lens, 1), ("parents", parents, 1), ("refs", refs, 1)):
        if not isinstance(t, torch.Tensor) or t.dim() != dims:
            raise OombError(ERR_INVALID_ARG, f"oomb_page_fork: {name} must be a tensor of {dims} dims")
    n_out, dev = int(parents.shape[0]), page_tables.device
    if tables_out is None:
        tables_out = torch.empty((n_out, page_tables.shape[1]), dtype=torch.int32, device=dev)
    if lens_out is None:
        lens_out = torch.empty((n_out,), dtype=torch.int32, device=dev)
    if refs_out is None:
        refs_out = refs
    if copies is None:
        copies = torch.empty((n_out, 3), dtype=torch.int32, device=dev)
    if status is None:
        status = torch.empty((2,), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = _workspace_of(page_fork_workspace_bytes(page_tables.shape[0], n_out, refs.shape[0]), dev)
    st = (_nb or _native()).page_fork(int(page_size), page_tables, seq_lens, parents, grow, refs, tables_out, lens_out, refs_out, copies, status, workspace)
    if st < 0:
        S, n_phys = _n(page_tables), _n(refs)
        raise _gen_refused("oomb_page_fork", [("page_tables", page_tables, (None, None)), ("seq_lens", seq_lens, (S,)), ("parents", parents, (n_out,)),
                                              ("grow", grow, (n_out,)), ("refs", refs, (None,)), ("tables_out", tables_out, (n_out, None)),
                                              ("lens_out", lens_out, (n_out,)), ("refs_out", refs_out, (n_phys,)), ("copies", copies, (n_out, 3)),
                                              ("status", status, (2,))], others=[("workspace", workspace)])
    if st != OK:
        raise OombError(st, "oomb_page_fork")
    return PageFork(tables_out, lens_out, refs_out, copies, status)


def page_compact_workspace_bytes(n_phys: int) -> int:
    """oomb_page_compact_workspace_bytes."""
    return int(lib().oomb_page_compact_workspace_bytes(int(n_phys)))


def page_compact(page_tables, seq_lens, refs, page_size: int, tables_out=None, refs_out=None, moves=None, page_map=None, status=None, workspace=None) -> PageCompact:
    """oomb_page_compact: the used pages renumbered to the lowest numbers.  page_tables and refs are updated in place unless others are given.
    page_copy(pools, result.moves, count=result.status[1:]) then moves what they hold."""
    for name, t, dims in (("page_tables", page_tables, 2), ("seq_lens", seq_lens, 1), ("refs", refs, 1)):
        if not isinstance(t, torch.Tensor) or t.dim() != dims:
            raise OombError(ERR_INVALID_ARG, f"oomb_page_compact: {name} must be a tensor of {dims} dims")
    n_phys, dev = int(refs.shape[0]), page_tables.device
    if tables_out is None:
        tables_out = page_tables
    if refs_out is None:
        refs_out = refs
    if moves is None:
        moves = torch.empty((max(1, n_phys // 2), 3), dtype=torch.int32, device=dev)
    if page_map is None:
        page_map = torch.empty((n_phys,), dtype=torch.int32, device=dev)
    if status is None:
        status = torch.empty((2,), dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = _workspace_of(page_compact_workspace_bytes(n_phys), dev)
    st = (_nb or _native()).page_compact(int(page_size), page_tables, seq_lens, refs, tables_out, refs_out, moves, page_map, status, workspace)
    if st < 0:
        raise _gen_refused("oomb_page_compact", [("page_tables", page_tables, (None, None)), ("seq_lens", seq_lens, (_n(page_tables),)), ("refs", refs, (None,)),
                                                 ("tables_out", tables_out, (_n(page_tables), _n(page_tables, 1))), ("refs_out", refs_out, (n_phys,)),
                                                 ("moves", moves, (None, 3)), ("page_map", page_map, (n_phys,)), ("status", status, (2,))],
                           others=[("workspace", workspace)])
    if st != OK:
        raise OombError(st, "oomb_page_compact")
    return PageCompact(tables_out, refs_out, moves, page_map, status)


def page_copy(pools, copies, count=None) -> None:
    """oomb_page_copy: the listed pages ([n][3] int32: source, destination, tokens) in every pool of a list: [n_phys][Hkv][P][D] of one shape, type
    and strides, or kvq_pools.  count [1] int32 on the device: how many of the list (default: all)."""
    if isinstance(pools, torch.Tensor):
        pools = (pools,)
    st = (_nb or _native()).page_copy(pools, copies, count)
    if st < 0:
        where = "oomb_page_copy"
        pools = list(pools)
        if not pools or any(not isinstance(t, torch.Tensor) or t.dim() not in (3, 4) or t.shape != pools[0].shape or t.stride() != pools[0].stride() or
                            t.dtype != pools[0].dtype or t.stride(-1) != 1 or (t.dim() == 3 and t.dtype != torch.uint8) for t in pools):
            raise OombError(ERR_INVALID_ARG, f"{where}: pools must be [n_phys][Hkv][P][D] (or kvq_pools) of one shape, type and strides")
        raise _gen_refused(where, [("copies", copies, (None, 3)), ("count", count, (1,))], others=[("pool", t) for t in pools])
    if st != OK:
        raise OombError(st, "oomb_page_copy")


def _beam_desc(logits, groups: int, n_out: int, pad_token: int = 0) -> BeamDesc:
    if not isinstance(logits, torch.Tensor) or logits.dim() not in (2, 3) or logits.dtype not in (torch.float32, torch.bfloat16) or \
            groups <= 0 or logits.shape[:-1].numel() % groups:
        raise OombError(ERR_INVALID_ARG, "oomb_beam_topk: logits must be [groups * beams][vocab] (or [groups][beams][vocab]) float32 or bfloat16")
    rows = logits.shape[:-1].numel()
    return BeamDesc(groups, rows // groups, int(logits.shape[-1]), int(n_out), _dt(logits.dtype), int(pad_token), logits.stride(-2) if rows > 1 else logits.shape[-1])


def beam_workspace_bytes(logits, groups: int, n_out: int) -> int:
    """oomb_beam_workspace_bytes."""
    return int(lib().oomb_beam_workspace_bytes(ctypes.byref(_beam_desc(logits, int(groups), n_out))))


def beam_topk(logits, scores, n_out: int, done=None, pad_token: int = 0, parents=None, tokens=None, scores_out=None, workspace=None):
    """oomb_beam_topk: of every group the n_out best continuations of its beams.  logits [groups * beams][vocab] or [groups][beams][vocab]; scores
    [groups][beams] float32; done [groups][beams] int32 (of the next step: the parents', and 1 where a token ends its
    text).  Returns (parents [groups][n_out] int32 rows of logits, tokens int32, scores float32)."""
    if not isinstance(scores, torch.Tensor) or scores.dim() != 2 or not isinstance(logits, torch.Tensor):
        raise OombError(ERR_INVALID_ARG, "oomb_beam_topk: scores must be float32 [groups][beams]")
    groups, dev = int(scores.shape[0]), logits.device
    if logits.dim() == 3:
        if logits.shape[0] != groups or (logits.shape[0] > 1 and logits.shape[1] > 1 and logits.stride(0) != logits.shape[1] * logits.stride(1)):
            raise OombError(ERR_INVALID_ARG, "oomb_beam_topk: logits [groups][beams][vocab] must have rows at equal distances")
        logits = logits.flatten(0, 1)
    desc = _beam_desc(logits, groups, n_out, pad_token)
    if parents is None:
        parents = torch.empty((groups, n_out), dtype=torch.int32, device=dev)
    if tokens is None:
        tokens = torch.empty((groups, n_out), dtype=torch.int32, device=dev)
    if scores_out is None:
        scores_out = torch.empty((groups, n_out), dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = _workspace_of(int(lib().oomb_beam_workspace_bytes(ctypes.byref(desc))), dev)
    st = (_nb or _native()).beam_topk(desc, logits, scores, done, parents, tokens, scores_out, workspace)
    if st < 0:
        W = desc.n_beams
        if logits.stride(-1) != 1 and logits.shape[-1] > 1:
            raise OombError(ERR_INVALID_ARG, "oomb_beam_topk: the vocabulary of logits must be contiguous")
        raise _gen_refused("oomb_beam_topk", [("done", done, (groups, W)), ("parents", parents, (groups, n_out)), ("tokens", tokens, (groups, n_out))],
                           [("scores", scores, (groups, W)), ("scores_out", scores_out, (groups, n_out))], [("logits", logits), ("workspace", workspace)])
    if st != OK:
        raise OombError(st, "oomb_beam_topk")
    return parents, tokens, scores_out
