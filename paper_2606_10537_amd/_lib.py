"""ctypes binding of ``libpd.so`` (the C ABI declared in include/pd.h).

Argument marshalling only: torch tensors are passed as device pointers, the
stream as its ``hipStream_t`` handle; every step of the path runs in the HIP
kernels.  If the library is missing this module raises -- there is no CPU
fallback.
"""

import ctypes
import os
from dataclasses import dataclass

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libpd.so")

PD_BF16, PD_FP32, PD_FP8_E4M3 = 0, 1, 2
STATUS = {0: "PD_OK", 1: "PD_ERR_NULL_PTR", 2: "PD_ERR_BAD_DIMS", 3: "PD_ERR_UNSUPPORTED",
          4: "PD_ERR_MISALIGNED", 5: "PD_ERR_WORKSPACE", 6: "PD_ERR_HIP"}

EXPORTS = ["pd_prefill_chunks", "pd_score_select", "pd_sparse_decode_attn", "pd_cache_bytes",
           "pd_workspace_bytes", "pd_decode_splits", "pd_status_string", "pd_last_error_message",
           "pd_version", "pd_mfma_rate_probe", "pd_score_select_static", "pd_gather_selected",
           "pd_sparse_decode_attn_compact", "pd_compact_workspace_bytes", "pd_select_ranked",
           "pd_gather_joint", "pd_score_select_noalloc", "pd_qk_norm_rope", "pd_paged_append", "pd_paged_read",
           "pd_paged_select", "pd_paged_attn", "pd_paged_workspace_bytes"]


class PdError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class PdDims(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_chunks", ctypes.c_int32), ("chunk_len", ctypes.c_int32),
        ("q_len", ctypes.c_int32), ("m_len", ctypes.c_int32), ("dec_len", ctypes.c_int32),
        ("n_heads_q", ctypes.c_int32), ("n_heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("sm_scale", ctypes.c_float), ("qm_per_chunk", ctypes.c_int32),
        ("out_fp32", ctypes.c_int32), ("tok_score_dir", ctypes.c_int32),
    ]


@dataclass
class Dims:
    """Problem sizes in the paper's notation (Section 5): B, N, C, L_q, L_m, L_d, heads, d."""
    batch: int
    n_chunks: int
    chunk_len: int
    q_len: int
    m_len: int
    dec_len: int
    n_heads_q: int
    n_heads_kv: int
    head_dim: int
    dtype: int = PD_BF16
    sm_scale: float = 0.0
    qm_per_chunk: int = 0
    out_fp32: int = 0
    tok_score_dir: int = 0

    @property
    def seq_len(self):
        """S_c = 1 + C + L_q + L_m, rows of one chunk sequence."""
        return 1 + self.chunk_len + self.q_len + self.m_len

    def c(self):
        return PdDims(self.batch, self.n_chunks, self.chunk_len, self.q_len, self.m_len, self.dec_len,
                      self.n_heads_q, self.n_heads_kv, self.head_dim, self.dtype, self.sm_scale,
                      self.qm_per_chunk, self.out_fp32, self.tok_score_dir)


class PagedDims(ctypes.Structure):
    """Sizes of a paged cache and of the calls on it (see pd_paged_dims in include/pd.h); built with keywords."""
    _fields_ = [
        ("batch", ctypes.c_int32), ("new_len", ctypes.c_int32), ("n_heads_q", ctypes.c_int32),
        ("n_heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("cache_dtype", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("n_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32), ("sm_scale", ctypes.c_float), ("causal", ctypes.c_int32),
    ]


class PdPagedCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "k_exp", "v_exp", "k_bounds", "page_table",
                                               "kv_len", "new_rows")]


_lib = None


def load(path: str = LIB_PATH):
    """Load libpd.so once and declare the signatures; raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"HIP library not built: {path} (run __graft_entry__.build())")
    # torch ships its own HIP runtime with the same soname; loading torch first
    # makes libpd.so bind to that one copy, so streams and device pointers the
    # caller gets from torch belong to the runtime that launches the kernels.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    vp, sz, i32, fp = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_void_p
    dp = ctypes.POINTER(PdDims)
    lib.pd_prefill_chunks.argtypes = [dp] + [vp] * 13 + [vp, sz, vp]
    lib.pd_prefill_chunks.restype = ctypes.c_int
    lib.pd_score_select.argtypes = [dp, i32, i32, vp, fp, fp, vp, vp, fp, vp, sz, vp]
    lib.pd_score_select.restype = ctypes.c_int
    lib.pd_sparse_decode_attn.argtypes = [dp, i32, i32] + [vp] * 9 + [i32, vp, fp, i32, vp, sz, vp]
    lib.pd_sparse_decode_attn.restype = ctypes.c_int
    lib.pd_cache_bytes.argtypes = [dp]
    lib.pd_cache_bytes.restype = sz
    lib.pd_workspace_bytes.argtypes = [dp, i32, i32, i32, i32]
    lib.pd_workspace_bytes.restype = sz
    lib.pd_decode_splits.argtypes = [dp, i32, i32, i32, i32]
    lib.pd_decode_splits.restype = i32
    lib.pd_status_string.argtypes = [ctypes.c_int]
    lib.pd_status_string.restype = ctypes.c_char_p
    lib.pd_last_error_message.argtypes = []
    lib.pd_last_error_message.restype = ctypes.c_char_p
    lib.pd_select_ranked.argtypes = [dp, i32, i32, fp, i32, fp, vp, vp, vp]
    lib.pd_select_ranked.restype = ctypes.c_int
    lib.pd_score_select_noalloc.argtypes = [dp, i32, i32, vp, fp, fp, vp, vp, fp, vp]
    lib.pd_score_select_noalloc.restype = ctypes.c_int
    lib.pd_score_select_static.argtypes = [dp, i32, i32, vp, fp, fp, vp, vp, fp, vp, sz, vp]
    lib.pd_score_select_static.restype = ctypes.c_int
    lib.pd_gather_selected.argtypes = [dp, i32, i32] + [vp] * 6 + [vp]
    lib.pd_gather_selected.restype = ctypes.c_int
    lib.pd_gather_joint.argtypes = [dp, i32, i32] + [vp] * 8 + [ctypes.c_double] + [vp] * 6
    lib.pd_gather_joint.restype = ctypes.c_int
    lib.pd_sparse_decode_attn_compact.argtypes = [dp, i32] + [vp] * 7 + [i32, vp, fp, i32, vp, sz, vp]
    lib.pd_sparse_decode_attn_compact.restype = ctypes.c_int
    lib.pd_compact_workspace_bytes.argtypes = [dp, i32, i32]
    lib.pd_compact_workspace_bytes.restype = sz
    lib.pd_mfma_rate_probe.argtypes = [i32, i32, vp, vp]
    lib.pd_mfma_rate_probe.restype = ctypes.c_int
    pp, cp, i64 = ctypes.POINTER(PagedDims), ctypes.POINTER(PdPagedCache), ctypes.c_int64
    lib.pd_qk_norm_rope.argtypes = [i32] * 5 + [vp, i64, vp, i64, vp, vp, ctypes.c_float, vp, ctypes.c_double,
                                                vp, i64, vp, i64, vp]
    lib.pd_qk_norm_rope.restype = ctypes.c_int
    lib.pd_paged_append.argtypes = [pp, cp, vp, i64, vp, i64, vp]
    lib.pd_paged_append.restype = ctypes.c_int
    lib.pd_paged_read.argtypes = [pp, cp, i32, i32, vp, vp, vp]
    lib.pd_paged_read.restype = ctypes.c_int
    lib.pd_paged_select.argtypes = [pp, cp, vp, i32, i32, i32, vp, vp, sz, vp]
    lib.pd_paged_select.restype = ctypes.c_int
    lib.pd_paged_attn.argtypes = [pp, cp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.pd_paged_attn.restype = ctypes.c_int
    lib.pd_paged_workspace_bytes.argtypes = [pp, i32, i32]
    lib.pd_paged_workspace_bytes.restype = sz
    lib.pd_version.argtypes = []
    lib.pd_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _ptr(t):
    """Device pointer of a tensor (or None / an int address)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors passed to the HIP library must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(status):
    if status != 0:
        raise PdError(status, load().pd_last_error_message().decode())


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def pd_cache_bytes(dims: Dims) -> int:
    return load().pd_cache_bytes(ctypes.byref(dims.c()))


def pd_workspace_bytes(dims: Dims, top_k=0, tok_budget=0, num_splits=0, which=0) -> int:
    return load().pd_workspace_bytes(ctypes.byref(dims.c()), top_k, tok_budget, num_splits, which)


def pd_decode_splits(dims: Dims, top_k, tok_budget, n_static, num_splits=0) -> int:
    return load().pd_decode_splits(ctypes.byref(dims.c()), top_k, tok_budget, n_static, num_splits)


def pd_prefill_chunks(dims: Dims, q_pre, k_pre, v_pre, q_qm, k_qm, v_qm, o, k_cache, v_cache,
                      tok_score, tok_rank, key_mean, workspace, stream=None, chunk_score=None):
    """Stage (a) for one layer (see include/pd.h); chunk_score (B, N) fp32 or None."""
    _check(load().pd_prefill_chunks(
        ctypes.byref(dims.c()), _ptr(q_pre), _ptr(k_pre), _ptr(v_pre), _ptr(q_qm), _ptr(k_qm), _ptr(v_qm),
        _ptr(o), _ptr(k_cache), _ptr(v_cache), _ptr(tok_score), _ptr(tok_rank), _ptr(key_mean),
        _ptr(chunk_score), _ptr(workspace), _nbytes(workspace), _stream(stream)))


def pd_select_ranked(dims: Dims, top_k, tok_budget, chunk_score, lowest, tok_rank, chunk_idx, tok_slot,
                     stream=None):
    """Top-K chunks by given scores (the lowest when lowest=1) and their kept tokens (see include/pd.h)."""
    _check(load().pd_select_ranked(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(chunk_score), int(lowest), _ptr(tok_rank),
        _ptr(chunk_idx), _ptr(tok_slot), _stream(stream)))


def pd_score_select(dims: Dims, top_k, tok_budget, q_dec, key_mean, tok_rank, chunk_idx, tok_slot,
                    chunk_score, workspace, stream=None):
    """Stage (b) for one layer and step (see include/pd.h)."""
    _check(load().pd_score_select(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(q_dec), _ptr(key_mean), _ptr(tok_rank),
        _ptr(chunk_idx), _ptr(tok_slot), _ptr(chunk_score), _ptr(workspace), _nbytes(workspace),
        _stream(stream)))


def pd_score_select_noalloc(dims: Dims, top_k, tok_budget, q_dec, key_mean, tok_rank, chunk_idx, tok_slot,
                            chunk_score=None, stream=None):
    """Stage (b) without a workspace: scratch in the library's static per-GPU array (see include/pd.h)."""
    _check(load().pd_score_select_noalloc(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(q_dec), _ptr(key_mean), _ptr(tok_rank),
        _ptr(chunk_idx), _ptr(tok_slot), _ptr(chunk_score), _stream(stream)))


def pd_sparse_decode_attn(dims: Dims, top_k, tok_budget, q_dec, k_dec, v_dec, k_cache, v_cache,
                          chunk_idx, tok_slot, k_static, v_static, n_static, o_dec, lse_dec,
                          num_splits, workspace, stream=None):
    """Stage (c) for one layer and step (see include/pd.h)."""
    _check(load().pd_sparse_decode_attn(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(q_dec), _ptr(k_dec), _ptr(v_dec),
        _ptr(k_cache), _ptr(v_cache), _ptr(chunk_idx), _ptr(tok_slot), _ptr(k_static), _ptr(v_static),
        n_static, _ptr(o_dec), _ptr(lse_dec), num_splits, _ptr(workspace), _nbytes(workspace),
        _stream(stream)))


def pd_score_select_static(dims: Dims, top_k, tok_budget, q_qm, key_mean, tok_rank, chunk_idx, tok_slot,
                           chunk_score, workspace, stream=None):
    """Static-selection mode: selection from the pseudo-label rows of q_qm (see include/pd.h)."""
    _check(load().pd_score_select_static(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(q_qm), _ptr(key_mean), _ptr(tok_rank),
        _ptr(chunk_idx), _ptr(tok_slot), _ptr(chunk_score), _ptr(workspace), _nbytes(workspace),
        _stream(stream)))


def pd_gather_selected(dims: Dims, top_k, tok_budget, k_cache, v_cache, chunk_idx, tok_slot, k_sel, v_sel,
                       stream=None):
    """Static-selection mode: copy the kept rows into contiguous buffers (see include/pd.h)."""
    _check(load().pd_gather_selected(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(k_cache), _ptr(v_cache), _ptr(chunk_idx),
        _ptr(tok_slot), _ptr(k_sel), _ptr(v_sel), _stream(stream)))


def pd_gather_joint(dims: Dims, top_k, tok_budget, chunk_idx, tok_slot, q_pre, k_cache, v_cache, q_qm, k_qm,
                    v_qm, rope_base, q_joint, k_joint, v_joint, k_pref=None, v_pref=None, stream=None):
    """Full-mask mode: joint rows [kept rows ; query rows] at continuous positions (see include/pd.h)."""
    _check(load().pd_gather_joint(
        ctypes.byref(dims.c()), top_k, tok_budget, _ptr(chunk_idx), _ptr(tok_slot), _ptr(q_pre), _ptr(k_cache),
        _ptr(v_cache), _ptr(q_qm), _ptr(k_qm), _ptr(v_qm), float(rope_base), _ptr(q_joint), _ptr(k_joint),
        _ptr(v_joint), _ptr(k_pref), _ptr(v_pref), _stream(stream)))


def pd_sparse_decode_attn_compact(dims: Dims, n_sel, q_dec, k_dec, v_dec, k_sel, v_sel, k_static, v_static,
                                  n_static, o_dec, lse_dec, num_splits, workspace, stream=None):
    """Stage (c) over a compact prefix buffer (see include/pd.h)."""
    _check(load().pd_sparse_decode_attn_compact(
        ctypes.byref(dims.c()), n_sel, _ptr(q_dec), _ptr(k_dec), _ptr(v_dec), _ptr(k_sel), _ptr(v_sel),
        _ptr(k_static), _ptr(v_static), n_static, _ptr(o_dec), _ptr(lse_dec), num_splits, _ptr(workspace),
        _nbytes(workspace), _stream(stream)))


def pd_compact_workspace_bytes(dims: Dims, n_sel, num_splits=0) -> int:
    return load().pd_compact_workspace_bytes(ctypes.byref(dims.c()), n_sel, num_splits)


def pd_mfma_rate_probe(n_workgroups, iters, sink, stream=None):
    """Launch the MFMA-rate diagnostic (n_workgroups * 4 * iters * 8 * 32768 FLOP)."""
    _check(load().pd_mfma_rate_probe(n_workgroups, iters, _ptr(sink), _stream(stream)))


# --------------------------------------------------------------------------- paged cache
# Sequences of these calls grow and shrink between calls, so the tensors' types, sizes and
# device are checked here against the sizes that the kernels will index by.  A call of one
# token takes the GPU a few microseconds, so what fits is told first, in a few comparisons,
# and the reason is looked for only where something does not.

_TYPES, _KINDS = {}, {}
_FAR = 1 << 31


def _torch():
    """torch, and the element types by pd_dtype and back, filled in once (loading the library imports it first)."""
    import torch
    if not _TYPES:
        # The table that is asked for above comes last: a thread that finds it filled needs both.
        _KINDS.update({torch.bfloat16: PD_BF16, torch.float32: PD_FP32, "int32": torch.int32, "uint8": torch.uint8})
        _TYPES.update({PD_BF16: torch.bfloat16, PD_FP32: torch.float32, PD_FP8_E4M3: torch.float8_e4m3fn})
    return torch


def _launch_stream(stream, device):
    """The stream's handle; the current stream of `device`, which has to be the current one, where none is given."""
    import torch
    if device != torch.cuda.current_device():
        raise ValueError(f"tensors on cuda:{device} while cuda:{torch.cuda.current_device()} is current")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    return _stream(stream)


def _refuse(name, t, shape, type_, device):
    if t.dtype is not type_:
        raise ValueError(f"{name} has type {t.dtype}, wanted {type_}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, wanted {tuple(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    raise ValueError(f"{name} is on cuda:{t.get_device()}, the call's other tensors on cuda:{device}")


def _checked(name, t, shape, type_, device):
    """Device pointer of a contiguous tensor of this shape and type on `device`."""
    if t.dtype is not type_ or t.shape != shape or t.get_device() != device:
        _refuse(name, t, shape, type_, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(name, t, shape, type_, device):
    """Pointer and row stride of a tensor [..., heads, d] whose heads lie one after another in a row and whose rows
    (all dimensions before the heads) lie one stride apart."""
    if t.dtype is not type_ or t.shape != shape or t.get_device() != device:
        _refuse(name, t, shape, type_, device)
    heads, d = shape[-2], shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), heads * d
    strides = t.stride()
    if (d > 1 and strides[-1] != 1) or (heads > 1 and strides[-2] != d):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    lead = [(n, s) for n, s in zip(shape[:-2], strides[:-2]) if n != 1]
    stride = want = lead[-1][1] if lead else heads * d
    for n, s in reversed(lead):
        if s != want:
            raise ValueError(f"{name}: its rows must lie one stride apart")
        want = n * s
    return t.data_ptr(), stride


def _space(workspace, device):
    """Pointer and size of a workspace, or of none."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != device:
        raise ValueError(f"the workspace is not on cuda:{device}, as the call's other tensors")
    return _ptr(workspace), _nbytes(workspace)


class PagedCache:
    """The tensors of a paged cache (see pd_paged_cache in include/pd.h), checked against `dims` once and kept alive.

    k_pages, v_pages [n_pages][H_kv][R][d]; page_table int32 [B][max_pages]; kv_len, new_rows int32 [B]; k_exp, v_exp
    uint8 [n_pages][H_kv][R] for PD_FP8_E4M3; k_bounds [n_pages][H_kv][2][d].  Calls may bring dims of their own that
    differ in new_len, n_heads_q, sm_scale and causal."""

    def __init__(self, dims, k_pages, v_pages, page_table, kv_len, new_rows=None, k_exp=None, v_exp=None,
                 k_bounds=None):
        torch = _torch()
        d = dims
        if not k_pages.is_cuda:
            raise ValueError("k_pages must be on the GPU")
        if d.dtype not in (PD_BF16, PD_FP32) or d.cache_dtype not in _TYPES:
            raise ValueError(f"no element type {d.dtype} or cache type {d.cache_dtype}")
        self.device = k_pages.get_device()
        self._key = self._sizes(dims)
        self.tensors = (k_pages, v_pages, k_exp, v_exp, k_bounds, page_table, kv_len, new_rows)
        if (d.cache_dtype == PD_FP8_E4M3) != (k_exp is not None) or (k_exp is None) != (v_exp is None):
            raise ValueError("k_exp and v_exp belong to a cache of PD_FP8_E4M3, and only to it")
        self.type = _TYPES[d.dtype]
        # E4M3 pages may also come as the bytes that they are.
        page = k_pages.dtype if d.cache_dtype == PD_FP8_E4M3 and k_pages.dtype is torch.uint8 else _TYPES[d.cache_dtype]
        pool = (d.n_pages, d.n_heads_kv, d.page_rows)
        wanted = ((pool + (d.head_dim,), page), (pool + (d.head_dim,), page), (pool, torch.uint8), (pool, torch.uint8),
                  (pool[:2] + (2, d.head_dim), self.type), ((d.batch, d.max_pages), torch.int32),
                  ((d.batch,), torch.int32), ((d.batch,), torch.int32))
        self.c = PdPagedCache()
        for (name, _), t, (shape, type_) in zip(PdPagedCache._fields_, self.tensors, wanted):
            if t is not None:
                setattr(self.c, name, _checked(name, t, shape, type_, self.device))
        self._ref = ctypes.byref(self.c)

    @staticmethod
    def _sizes(dims):
        """What of the sizes belongs to the pool and the batch: batch, and n_heads_kv .. max_pages."""
        raw = bytes(dims)
        return raw[:4] + raw[12:40]

    def _for(self, dims):
        if self._sizes(dims) != self._key:
            raise ValueError("dims differ from those that the cache was made with")
        return self._ref


def pd_qk_norm_rope(q, k, w_q, w_k, eps, pos, rope_base, q_out, k_out, stream=None):
    """Head norms and rotary positions of q [T, H_q, d] and k [T, H_kv, d] (see include/pd.h); rows may be strided;
    k and k_out None: queries alone; w_q, w_k None: no norm; rope_base 0: no rotation."""
    _torch()
    type_, shape, device = q.dtype, q.shape, q.get_device()
    if type_ not in _KINDS or len(shape) != 3 or device < 0:
        raise ValueError(f"q must be [rows, heads, d] in bf16 or fp32 on the GPU, got {tuple(shape)} {type_} {q.device}")
    T, hq, d = shape
    qp, qs = _rows("q", q, shape, type_, device)
    qo, qos = _rows("q_out", q_out, shape, type_, device)
    hkv, kp, ks, ko, kos = 0, None, 0, None, 0
    if k is not None:
        hkv = k.shape[1] if k.dim() == 3 else 0
        kp, ks = _rows("k", k, (T, hkv, d), type_, device)
        ko, kos = _rows("k_out", k_out, (T, hkv, d), type_, device)
    wq = None if w_q is None else _checked("w_q", w_q, (d,), type_, device)
    wk = None if w_k is None else _checked("w_k", w_k, (d,), type_, device)
    pp = None if pos is None else _checked("pos", pos, (T,), _KINDS["int32"], device)
    _check(load().pd_qk_norm_rope(T, hq, hkv, d, _KINDS[type_], qp, qs, kp, ks, wq, wk, eps, pp, rope_base,
                                  qo, qos, ko, kos, _launch_stream(stream, device)))


def pd_paged_workspace_bytes(dims: PagedDims, top_k=0, which=1) -> int:
    if not -_FAR <= top_k < _FAR or not -_FAR <= which < _FAR:   # ctypes would keep the low 32 bits
        raise ValueError(f"top_k={top_k} and which={which} must fit 32 bits")
    return load().pd_paged_workspace_bytes(ctypes.byref(dims), top_k, which)


def pd_paged_append(dims: PagedDims, cache: PagedCache, k_new, v_new, stream=None):
    """New rows k_new, v_new [B, L_n, H_kv, d] into the pages (see include/pd.h); rows may be strided."""
    shape, c, dev = (dims.batch, dims.new_len, dims.n_heads_kv, dims.head_dim), cache._for(dims), cache.device
    kp, ks = _rows("k_new", k_new, shape, cache.type, dev)
    vp, vs = _rows("v_new", v_new, shape, cache.type, dev)
    _check(load().pd_paged_append(ctypes.byref(dims), c, kp, ks, vp, vs, _launch_stream(stream, dev)))


def pd_paged_read(dims: PagedDims, cache: PagedCache, first, n_rows, k_out, v_out, stream=None):
    """Positions first..first+n_rows-1 of every sequence into k_out, v_out [B, H_kv, n_rows, d] (see include/pd.h)."""
    shape, c, dev = (dims.batch, dims.n_heads_kv, n_rows, dims.head_dim), cache._for(dims), cache.device
    if not -_FAR <= first < _FAR:
        raise ValueError(f"first={first} must fit 32 bits")
    _check(load().pd_paged_read(ctypes.byref(dims), c, first, n_rows, _checked("k_out", k_out, shape, cache.type, dev),
                                _checked("v_out", v_out, shape, cache.type, dev), _launch_stream(stream, dev)))


def pd_paged_select(dims: PagedDims, cache: PagedCache, q, top_k, n_first, n_last, page_idx, workspace, stream=None):
    """The top_k pages of each (sequence, KV head) by a bound on their scores (see include/pd.h)."""
    c, dev = cache._for(dims), cache.device
    if not -_FAR <= n_first < _FAR or not -_FAR <= n_last < _FAR:
        raise ValueError(f"n_first={n_first} and n_last={n_last} must fit 32 bits")
    qp = _checked("q", q, (dims.batch, dims.new_len, dims.n_heads_q, dims.head_dim), cache.type, dev)
    ip = _checked("page_idx", page_idx, (dims.batch, dims.n_heads_kv, top_k), _KINDS["int32"], dev)
    _check(load().pd_paged_select(ctypes.byref(dims), c, qp, top_k, n_first, n_last, ip, *_space(workspace, dev),
                                  _launch_stream(stream, dev)))


def pd_paged_attn(dims: PagedDims, cache: PagedCache, q, o, lse=None, page_idx=None, workspace=None, stream=None):
    """Attention of the new rows q [B, L_n, H_q, d] over the pages, or over those of page_idx [B, H_kv, K] (see
    include/pd.h); lse [B, H_q, L_n] fp32 or None."""
    c, dev = cache._for(dims), cache.device
    B, L, hq = dims.batch, dims.new_len, dims.n_heads_q
    shape, top_k, ip = (B, L, hq, dims.head_dim), 0, None
    if page_idx is not None:
        top_k = page_idx.shape[-1]
        if top_k < 1:   # a tensor without elements may have no address, which would mean all pages
            raise ValueError("page_idx has no entries; without a list (None) all pages are attended to")
        ip = _checked("page_idx", page_idx, (B, dims.n_heads_kv, top_k), _KINDS["int32"], dev)
    lp = None if lse is None else _checked("lse", lse, (B, hq, L), _TYPES[PD_FP32], dev)
    _check(load().pd_paged_attn(ctypes.byref(dims), c, _checked("q", q, shape, cache.type, dev), ip, top_k,
                                _checked("o", o, shape, cache.type, dev), lp, *_space(workspace, dev),
                                _launch_stream(stream, dev)))
