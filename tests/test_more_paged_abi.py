"""Refusals of pd_paged_window_attn, pd_paged_append_rope and of caches in 4 bits, on the host (nothing is launched; the
pointers are fake), the sizes of workspaces, and the binding's own checks of tensors."""

import ctypes
import math

import pytest
import torch

from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP4_E2M1, PD_FP8_E4M3
from test_paged_abi import A, ALIGN, BAD, DIMS, MIS, NULL, UNSUP, WS, append, attn, cache, dims, lib, read  # noqa: F401


def window(lib, d=None, c=None, q=A, w=100, s=4, o=A, lse=None, ws=A, n=1 << 40):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_window_attn(ctypes.byref(d), ctypes.byref(c), q, w, s, o, lse, ws, n, None)


@pytest.mark.parametrize("kw,want", BAD, ids=[str(k) for k, _ in BAD])
def test_sizes(lib, kw, want):  # noqa: F811
    d = dims(**kw)
    assert window(lib, d) == want
    assert lib.pd_paged_window_workspace_bytes(ctypes.byref(d), 100, 4) == 0


def test_window_refusals(lib):  # noqa: F811
    assert window(lib, w=0) == DIMS and window(lib, w=-(1 << 31)) == DIMS and window(lib, s=-1) == DIMS
    d, c = dims(), cache()
    assert lib.pd_paged_window_attn(None, ctypes.byref(c), A, 1, 0, A, None, A, 0, None) == NULL
    assert lib.pd_paged_window_attn(ctypes.byref(d), None, A, 1, 0, A, None, A, 0, None) == NULL
    for name in ("k_pages", "v_pages", "page_table", "kv_len"):
        assert window(lib, c=cache(**{name: None})) == NULL and window(lib, c=cache(**{name: MIS})) == ALIGN
    assert window(lib, q=None) == NULL and window(lib, o=None) == NULL and window(lib, q=MIS) == ALIGN
    assert window(lib, lse=MIS) == ALIGN and window(lib, c=cache(new_rows=MIS)) == ALIGN
    need = lib.pd_paged_window_workspace_bytes(ctypes.byref(dims()), 2000, 0)
    assert need > 0 and window(lib, w=2000, s=0, n=need - 1) == WS and window(lib, w=2000, ws=None) == WS
    assert window(lib, w=2000, ws=MIS) == ALIGN
    huge = dims(batch=65536, n_heads_q=16384, n_heads_kv=16384, new_len=2, max_pages=1 << 24)
    assert window(lib, huge) == DIMS and lib.pd_paged_window_workspace_bytes(ctypes.byref(huge), 1, 0) == 0


def test_window_workspaces(lib):  # noqa: F811
    """They go by the window, at most by the table, and follow any 32-bit window."""
    size = lambda d, w, s=0: _lib.pd_paged_window_workspace_bytes(d, w, s)  # noqa: E731
    long, short = dims(max_pages=1 << 20), dims(max_pages=64)
    assert size(long, 1000) == size(short, 1000) > 0 and size(long, 1) == 0
    most = _lib.pd_paged_workspace_bytes(long, 0, 1)
    assert size(long, (1 << 31) - 1, (1 << 31) - 1) == most and size(dims(max_pages=1 << 24, page_rows=64), (1 << 31) - 1, 9) > 0
    for w in (0, -1, -(1 << 31)):
        assert size(long, w) == 0
    assert size(long, 5, -1) == 0
    for bad in (1 << 31, -(1 << 31) - 1):
        with pytest.raises(ValueError, match="32 bits"):
            size(long, bad)
        with pytest.raises(ValueError, match="32 bits"):
            size(long, 1, bad)


@pytest.mark.parametrize("call", [append, read, attn, window])
def test_four_bits(lib, call):  # noqa: F811
    """They go with bf16 rows alone, and need their exponent bytes."""
    assert call(lib, dims(dtype=PD_FP32, cache_dtype=PD_FP4_E2M1)) == UNSUP and call(lib, dims(cache_dtype=4)) == UNSUP
    assert call(lib, dims(dtype=PD_FP4_E2M1, cache_dtype=PD_FP4_E2M1)) == UNSUP
    for name in ("k_exp", "v_exp"):
        assert call(lib, dims(cache_dtype=PD_FP4_E2M1), cache(**{name: None})) == NULL
        assert call(lib, dims(cache_dtype=PD_FP4_E2M1), cache(**{name: MIS})) == ALIGN


class Fake(torch.Tensor):
    """A CPU tensor that says that it lies on cuda:0, for checks that come before any call of the library."""

    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def fake(*shape, dtype):
    return torch.zeros(shape, dtype=dtype).as_subclass(Fake)


def four(**kw):
    d = dims(cache_dtype=PD_FP4_E2M1, n_pages=3, max_pages=2, page_rows=16)
    t = dict(k_pages=fake(3, 2, 16, 64, dtype=torch.uint8), v_pages=fake(3, 2, 16, 64, dtype=torch.uint8),
             page_table=fake(2, 2, dtype=torch.int32), kv_len=fake(2, dtype=torch.int32),
             k_exp=fake(3, 2, 4, 16, dtype=torch.uint8), v_exp=fake(3, 2, 4, 16, dtype=torch.uint8))
    return d, _lib.PagedCache(d, **dict(t, **kw))


def test_binding_checks_a_cache_of_four_bits(lib):  # noqa: F811
    assert four()[1].type is torch.bfloat16
    for kw, text in ((dict(k_exp=None), "belong to a cache"), (dict(k_exp=None, v_exp=None), "belong to a cache"),
                     (dict(k_pages=fake(3, 2, 16, 128, dtype=torch.uint8)), "shape"),
                     (dict(v_pages=fake(3, 2, 16, 64, dtype=torch.int8)), "type"),
                     (dict(k_exp=fake(3, 2, 16, 4, dtype=torch.uint8)), "shape"),
                     (dict(v_exp=fake(3, 2, 16, dtype=torch.uint8)), "shape")):
        with pytest.raises(ValueError, match=text):
            four(**kw)


def test_binding_checks_window_calls(lib):  # noqa: F811
    d, c = four()
    q = fake(2, 1, 8, 128, dtype=torch.bfloat16)
    for kw, text in ((dict(q=q[:, :, :4]), "shape"), (dict(q=fake(2, 1, 8, 128, dtype=torch.float32)), "type"),
                     (dict(o=fake(2, 1, 8, 64, dtype=torch.bfloat16)), "shape"), (dict(window=1 << 31), "32 bits"),
                     (dict(n_sinks=-(1 << 31) - 1), "32 bits"), (dict(lse=fake(2, 1, 8, dtype=torch.float32)), "shape")):
        args = dict(dict(q=q, window=4, n_sinks=0, o=q, lse=None), **kw)
        with pytest.raises(ValueError, match=text):
            _lib.pd_paged_window_attn(d, c, **args)
    other = dims(cache_dtype=PD_FP8_E4M3, n_pages=3, max_pages=2, page_rows=16)
    with pytest.raises(ValueError, match="differ"):
        _lib.pd_paged_window_attn(other, c, q, 4, 0, q)


def rope(lib, d=None, c=None, q=A, qs=1024, k=A, ks=256, v=A, vs=256, wq=A, wk=A, eps=1e-6, pos=A, base=1e4, qo=A):
    d, c = d or dims(), c or cache()
    return lib.pd_paged_append_rope(ctypes.byref(d), ctypes.byref(c), q, qs, k, ks, v, vs, wq, wk, eps, pos, base, qo, None)


@pytest.mark.parametrize("kw,want", BAD, ids=[str(k) for k, _ in BAD])
def test_rope_sizes(lib, kw, want):  # noqa: F811
    assert rope(lib, dims(**kw), qs=1 << 24, ks=1 << 24, vs=1 << 24) == want


def test_rope_refusals(lib):  # noqa: F811
    d, c = dims(), cache()
    tail = (A, 1024, A, 256, A, 256, A, A, 1e-6, A, 1e4, A, None)
    assert lib.pd_paged_append_rope(None, ctypes.byref(c), *tail) == NULL
    assert lib.pd_paged_append_rope(ctypes.byref(d), None, *tail) == NULL
    for name in ("k_pages", "v_pages", "page_table", "kv_len"):
        assert rope(lib, c=cache(**{name: None})) == NULL and rope(lib, c=cache(**{name: MIS})) == ALIGN
    for cache_dtype in (PD_FP8_E4M3, PD_FP4_E2M1):
        for name in ("k_exp", "v_exp"):
            assert rope(lib, dims(cache_dtype=cache_dtype), cache(**{name: None})) == NULL
    assert rope(lib, c=cache(k_bounds=MIS)) == ALIGN and rope(lib, c=cache(new_rows=MIS)) == ALIGN
    for name in ("q", "k", "v", "qo"):                          # q and q_out go together
        assert rope(lib, **{name: None}) == NULL and rope(lib, **{name: MIS}) == ALIGN
    for name in ("wq", "wk", "pos"):
        assert rope(lib, **{name: MIS}) == ALIGN
    assert rope(lib, eps=-1.0) == DIMS and rope(lib, eps=math.nan) == DIMS and rope(lib, eps=math.inf) == DIMS
    assert rope(lib, base=-1.0) == DIMS and rope(lib, base=math.inf) == DIMS and rope(lib, base=math.nan) == DIMS
    for name, least in (("qs", 1024), ("ks", 256), ("vs", 256)):
        for bad in (least - 8, least + 4, (1 << 40) + 8, -(1 << 63)):
            assert rope(lib, **{name: bad}) == DIMS
    assert rope(lib, q=A, qo=A, qs=1032) == DIMS                 # in place, with gaps between the rows
    assert b"q_out" in lib.pd_last_error_message()
    huge = dims(batch=65536, n_heads_q=16384, n_heads_kv=16384, new_len=2, max_pages=1 << 24)
    assert rope(lib, huge, qs=1 << 21, ks=1 << 21, vs=1 << 21) == DIMS


def test_binding_checks_rope_calls(lib):  # noqa: F811
    d, c = four()
    fused = fake(2, 1, 12, 128, dtype=torch.bfloat16)
    good = dict(q=fused[:, :, :8], k_new=fused[:, :, 8:10], v_new=fused[:, :, 10:], w_q=fake(128, dtype=torch.bfloat16),
                w_k=None, eps=0.0, pos=fake(2, 1, dtype=torch.int32), rope_base=1e4,
                q_out=fake(2, 1, 8, 128, dtype=torch.bfloat16))
    for kw, text in ((dict(q=None), "together"), (dict(q_out=None), "together"), (dict(k_new=fused[:, :, 8:9]), "shape"),
                     (dict(v_new=fused[:, :, 10:].float()), "type"), (dict(w_q=fake(64, dtype=torch.bfloat16)), "shape"),
                     (dict(w_k=fake(128, dtype=torch.float32)), "type"), (dict(pos=fake(2, dtype=torch.int32)), "shape"),
                     (dict(pos=fake(2, 1, dtype=torch.int64)), "type"), (dict(q_out=fused[:, :, :8].expand(2, 1, 8, 128)[..., :64]), "shape"),
                     (dict(k_new=fused[:, :, 8:12:2]), "contiguous"), (dict(w_q=torch.zeros(128, dtype=torch.bfloat16)), "GPU")):
        with pytest.raises(ValueError, match=text):
            _lib.pd_paged_append_rope(d, c, **dict(good, **kw))


def test_rows_of_a_projection(lib):  # noqa: F811
    """The stride that the binding finds for a strided [B, L, heads, d] is that of every row; other layouts are refused."""
    g = torch.Generator().manual_seed(0)
    for _ in range(300):
        B, L, H, d, extra = (int(torch.randint(lo, hi, (), generator=g)) for lo, hi in ((1, 4), (1, 4), (1, 4), (1, 5), (0, 3)))
        t = torch.zeros(B, L, H + extra, d)[:, :, :H]
        ptr, stride = _lib._rows("t", t, (B, L, H, d), torch.float32, -1)
        assert ptr == t.data_ptr()
        for b in range(B):
            for r in range(L):
                assert t[b, r].data_ptr() == ptr + 4 * (b * L + r) * stride
    base = torch.zeros(4, 6, 8, 16)
    for bad in (base[:, ::2], base[:, :, ::2], base.transpose(1, 2), base[..., ::2], base[:, 1:4]):
        shape = tuple(bad.shape)
        if bad.is_contiguous():
            continue
        try:
            ptr, stride = _lib._rows("t", bad, shape, torch.float32, -1)
        except ValueError:
            continue
        for b in range(shape[0]):
            for r in range(shape[1]):
                assert bad[b, r].data_ptr() == ptr + 4 * (b * shape[1] + r) * stride
                assert bad[b, r].is_contiguous()
