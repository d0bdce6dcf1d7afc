"""Refusals of the paged-cache entry points, on the host: nothing is launched (the pointers are fake), and the binding's
own checks of tensors, on the CPU."""

import ctypes
import math

import pytest
import torch

from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3, PagedDims, PdPagedCache

A = 1 << 20
MIS = A + 8
NULL, DIMS, UNSUP, ALIGN, WS = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def dims(**kw):
    base = dict(batch=2, new_len=1, n_heads_q=8, n_heads_kv=2, head_dim=128, dtype=PD_BF16, cache_dtype=PD_BF16,
                page_rows=64, n_pages=100, max_pages=40, sm_scale=0.0, causal=1)
    return PagedDims(**dict(base, **kw))


def cache(**kw):
    c = PdPagedCache(k_pages=A, v_pages=A, k_exp=A, v_exp=A, k_bounds=A, page_table=A, kv_len=A, new_rows=None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def append(lib, d=None, c=None, k=A, ks=256, v=A, vs=256):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_append(ctypes.byref(d), ctypes.byref(c), k, ks, v, vs, None)


def read(lib, d=None, c=None, first=0, n=64, k=A, v=A):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_read(ctypes.byref(d), ctypes.byref(c), first, n, k, v, None)


def select(lib, d=None, c=None, q=A, k=4, first=0, last=0, idx=A, ws=A, n=1 << 30):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_select(ctypes.byref(d), ctypes.byref(c), q, k, first, last, idx, ws, n, None)


def attn(lib, d=None, c=None, q=A, idx=None, k=0, o=A, lse=None, ws=A, n=1 << 40):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_attn(ctypes.byref(d), ctypes.byref(c), q, idx, k, o, lse, ws, n, None)


BAD = [(dict(batch=0), DIMS), (dict(batch=65537), DIMS), (dict(new_len=0), DIMS), (dict(new_len=(1 << 24) + 1), DIMS),
       (dict(n_heads_q=0), DIMS), (dict(n_heads_kv=0), DIMS), (dict(n_heads_kv=3), UNSUP), (dict(head_dim=96), UNSUP),
       (dict(dtype=PD_FP8_E4M3), UNSUP), (dict(dtype=9), UNSUP), (dict(cache_dtype=PD_FP32), UNSUP),
       (dict(dtype=PD_FP32, cache_dtype=PD_FP8_E4M3), UNSUP), (dict(cache_dtype=-1), UNSUP), (dict(page_rows=8), DIMS),
       (dict(page_rows=48), DIMS), (dict(page_rows=512), DIMS), (dict(n_pages=0), DIMS), (dict(max_pages=0), DIMS),
       (dict(max_pages=(1 << 24) + 1), DIMS), (dict(sm_scale=math.inf), DIMS), (dict(causal=2), DIMS),
       (dict(batch=1 << 16, n_heads_q=1 << 15, n_heads_kv=1), DIMS)]


@pytest.mark.parametrize("kw,want", BAD, ids=[str(k) for k, _ in BAD])
def test_sizes(lib, kw, want):
    d = dims(**kw)
    assert append(lib, d, ks=1 << 24, vs=1 << 24) == want
    assert read(lib, d) == want
    assert select(lib, d) == want
    assert attn(lib, d) == want
    assert _lib.pd_paged_workspace_bytes(d, 0, 1) == 0 and _lib.pd_paged_workspace_bytes(d, 4, 0) == 0


def test_null_and_misaligned(lib):
    d, c = dims(), cache()
    for f in (lib.pd_paged_append,):
        assert f(None, ctypes.byref(c), A, 256, A, 256, None) == NULL
        assert f(ctypes.byref(d), None, A, 256, A, 256, None) == NULL
    for name in ("k_pages", "v_pages", "page_table", "kv_len"):
        for call in (append, read, attn):
            assert call(lib, c=cache(**{name: None})) == NULL
            assert call(lib, c=cache(**{name: MIS})) == ALIGN
    for name in ("k_exp", "v_exp"):
        for call in (append, read, attn):
            assert call(lib, dims(cache_dtype=PD_FP8_E4M3), cache(**{name: None})) == NULL
            assert call(lib, dims(cache_dtype=PD_FP8_E4M3), cache(**{name: MIS})) == ALIGN
    assert append(lib, c=cache(new_rows=MIS)) == ALIGN and append(lib, c=cache(k_bounds=MIS)) == ALIGN
    assert select(lib, c=cache(k_bounds=None)) == NULL
    assert b"k_bounds" in lib.pd_last_error_message()
    for kw in (dict(k=None), dict(v=None)):
        assert append(lib, **kw) == NULL and read(lib, **kw) == NULL
    for kw in (dict(k=MIS), dict(v=MIS)):
        assert append(lib, **kw) == ALIGN and read(lib, **kw) == ALIGN
    assert select(lib, q=None) == NULL and select(lib, idx=None) == NULL and select(lib, idx=MIS) == ALIGN
    assert attn(lib, q=None) == NULL and attn(lib, o=None) == NULL and attn(lib, lse=MIS) == ALIGN
    assert attn(lib, idx=MIS, k=4) == ALIGN


def test_strides_ranges_and_workspaces(lib):
    assert append(lib, ks=248) == DIMS and append(lib, vs=257) == DIMS and append(lib, ks=(1 << 40) + 8) == DIMS
    assert read(lib, first=-1) == DIMS and read(lib, n=0) == DIMS and read(lib, first=2500, n=61) == DIMS
    assert select(lib, k=0) == DIMS and select(lib, k=41) == DIMS and select(lib, first=-1) == DIMS
    assert select(lib, dims(max_pages=65537, page_rows=16), k=4) == DIMS
    need = _lib.pd_paged_workspace_bytes(dims(), 4, 0)
    assert need >= 2 * 2 * 40 * 8 and select(lib, n=need - 1) == WS and select(lib, ws=None) == WS
    assert select(lib, ws=MIS) == ALIGN
    assert attn(lib, idx=A, k=0) == DIMS and attn(lib, idx=A, k=41) == DIMS and attn(lib, idx=None, k=4) == DIMS
    need = _lib.pd_paged_workspace_bytes(dims(), 0, 1)
    assert need > 0 and attn(lib, n=need - 1) == WS and attn(lib, ws=None) == WS and attn(lib, ws=MIS) == ALIGN
    # A table of one block of keys: nothing is ever cut, no workspace.
    assert _lib.pd_paged_workspace_bytes(dims(max_pages=2), 0, 1) == 0
    assert _lib.pd_paged_workspace_bytes(dims(), 0, 2) == 0 and _lib.pd_paged_workspace_bytes(dims(), 41, 1) == 0


def norm(lib, T=4, hq=4, hkv=2, d=64, dt=PD_BF16, q=A, qs=256, k=A, ks=128, wq=A, wk=A, eps=1e-6, pos=A, base=1e4, qo=A,
         qos=256, ko=A, kos=128):
    return lib.pd_qk_norm_rope(T, hq, hkv, d, dt, q, qs, k, ks, wq, wk, eps, pos, base, qo, qos, ko, kos, None)


def test_norm_refusals(lib):
    assert norm(lib, T=-1) == DIMS and norm(lib, hq=-1) == DIMS and norm(lib, hq=0, hkv=0) == DIMS
    assert norm(lib, T=(1 << 31) - 1, hq=4, hkv=2) == DIMS
    assert norm(lib, d=32) == UNSUP and norm(lib, dt=PD_FP8_E4M3) == UNSUP
    assert norm(lib, eps=-1.0) == DIMS and norm(lib, eps=math.nan) == DIMS
    assert norm(lib, base=-1.0) == DIMS and norm(lib, base=math.inf) == DIMS
    for name in ("q", "k", "qo", "ko", "pos"):
        assert norm(lib, **{name: None}) == NULL and norm(lib, **{name: MIS}) == ALIGN
    assert norm(lib, wq=MIS) == ALIGN and norm(lib, wk=MIS) == ALIGN
    for name, least in (("qs", 256), ("ks", 128), ("qos", 256), ("kos", 128)):
        assert norm(lib, **{name: least - 8}) == DIMS and norm(lib, **{name: least + 4}) == DIMS
    assert norm(lib, T=0, q=None, k=None, qo=None, ko=None) == 0


def test_existing_calls_refuse_the_cache_type(lib):
    from test_abi import dims as chunk_dims, prefill
    assert prefill(chunk_dims(dtype=PD_FP8_E4M3)) == UNSUP


def test_binding_checks_tensors(lib):
    """Types, shapes, strides and places are refused before anything reaches the library."""
    d = dims(n_pages=3, max_pages=2, page_rows=16)
    k = torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        _lib.PagedCache(d, k, k, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    x = torch.zeros(4, 6, 64)
    with pytest.raises(ValueError, match="on the GPU"):
        _lib.pd_qk_norm_rope(x[:, :4], x[:, 4:], None, None, 0.0, None, 0.0, x[:, :4].clone(), x[:, 4:].clone())
    with pytest.raises(ValueError, match="bf16 or fp32"):
        _lib.pd_qk_norm_rope(x.double(), None, None, None, 0.0, None, 0.0, x.double(), None)
    types = torch.float32
    with pytest.raises(ValueError, match="type"):
        _lib._rows("x", x, x.shape, torch.bfloat16, -1)
    with pytest.raises(ValueError, match="shape"):
        _lib._rows("x", x, (4, 6, 32), types, -1)
    with pytest.raises(ValueError, match="heads of a row"):
        _lib._rows("x", x.transpose(0, 1), (6, 4, 64), types, -1)
    with pytest.raises(ValueError, match="one stride apart"):
        _lib._rows("x", torch.zeros(2, 5, 6, 64)[:, :4], (2, 4, 6, 64), types, -1)
    with pytest.raises(ValueError, match="contiguous"):
        _lib._checked("x", torch.zeros(6, 4).t(), (4, 6), types, -1)


def test_binding_types_are_complete_once_they_are_seen(lib, monkeypatch):
    """The element types are filled in at the first call; a thread that finds one table filled relies on the other."""
    kinds = {}

    class Watched(dict):
        def update(self, *a, **kw):
            super().update(*a, **kw)
            assert len(kinds) == 4, "another thread would take the tables for complete here"

    types = Watched()
    monkeypatch.setattr(_lib, "_KINDS", kinds)
    monkeypatch.setattr(_lib, "_TYPES", types)
    _lib._torch()
    assert len(types) == 3 and set(types.values()) >= {torch.bfloat16, torch.float32}


class _OnTheHost:
    """Stands for a PagedCache, so that the calls' checks run on CPU tensors (whose device number is -1)."""
    device, type = -1, torch.bfloat16

    def _for(self, dims):
        return ctypes.byref(cache())


def test_an_empty_list_of_pages_is_not_all_pages(lib):
    """page_idx of no entries has no address, which the library would take for no list at all: refused."""
    d = dims()
    q = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    idx = torch.zeros(2, 2, 0, dtype=torch.int32)
    assert idx.data_ptr() == 0
    with pytest.raises(ValueError, match="page_idx"):
        _lib.pd_paged_attn(d, _OnTheHost(), q, q.clone(), page_idx=idx)


@pytest.mark.parametrize("far", [1 << 31, 1 << 32, (1 << 32) + 7, -(1 << 32)])
def test_binding_refuses_numbers_beyond_32_bits(lib, far):
    """Position and page counts are 32 bits in the library; a larger number is refused, not cut to its low bits."""
    d = dims()
    q = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    out = torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16)
    idx = torch.zeros(2, 2, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="first"):
        _lib.pd_paged_read(d, _OnTheHost(), far, 64, out, out.clone())
    for first, last in ((far, 0), (0, far)):
        with pytest.raises(ValueError, match="n_first"):
            _lib.pd_paged_select(d, _OnTheHost(), q, 4, first, last, idx, None)
    for top_k, which in ((far, 1), (4, far)):
        with pytest.raises(ValueError, match="top_k"):
            _lib.pd_paged_workspace_bytes(d, top_k, which)
