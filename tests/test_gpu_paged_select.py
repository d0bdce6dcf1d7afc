"""pd_paged_select: the oracle's pages exactly, and pd_paged_attn over them."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged_case import Case, check_attn, h64, run_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

pytestmark = pytest.mark.gpu


def select(case, c, top_k, first, last):
    d = case.dims
    out = torch.full((d.batch, d.n_heads_kv, top_k), 99, dtype=torch.int32, device="cuda")
    ws = torch.full((_lib.pd_paged_workspace_bytes(d, top_k, 0),), 255, dtype=torch.uint8, device="cuda")
    _lib.pd_paged_select(d, c["cache"], c["q"], top_k, first, last, out, ws)
    return out


def want(case, top_k, first, last):
    d = case.dims
    out = np.full((d.batch, d.n_heads_kv, top_k), -1)
    bounds = h64(case.pool["bounds"])
    for b in range(d.batch):
        pages = -(-case.lens[b] // d.page_rows)
        idx = case.table[b, :pages].long().numpy()
        for g in range(d.n_heads_kv):
            q = case.rows_of(b, g)
            lo, hi = bounds[idx, g, 0], bounds[idx, g, 1]
            s = ref.page_scores_ref(q, lo, hi) if len(q) and pages else np.full(pages, -np.inf)
            best = ref.select_ref(s, top_k, first, last)
            out[b, g, :len(best)] = best
    return out


@pytest.mark.parametrize("dtype,cache", [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)])
@pytest.mark.parametrize("hq,hkv,d,R,L,lens,k,first,last", [
    (4, 2, 64, 16, 1, [200, 16, 0, 1, 500], 5, 1, 2), (8, 1, 128, 16, 1, [3000], 17, 0, 0),
    (6, 3, 128, 32, 3, [700, 90], 4, 0, 1), (34, 2, 64, 16, 2, [260, 250], 3, 2, 2), (1, 1, 64, 16, 1, [64], 4, 9, 9),
    (8, 1, 128, 16, 33, [300, 40, 33], 6, 0, 1), (12, 2, 64, 16, 9, [5000, 100], 40, 1, 0)])
def test_pages_and_their_attention(gpu_lib, dtype, cache, hq, hkv, d, R, L, lens, k, first, last):
    print(f"[select] {dtype}/{cache} {hq}/{hkv} d={d} R={R} L={L} {lens} top {k}", flush=True)
    new = [min(L, n) for n in lens]
    case = Case(lens, new_len=L, new=new, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, R=R, seed=k)
    c = case.to_gpu()
    k = min(k, case.dims.max_pages)
    got = select(case, c, k, first, last)
    assert np.array_equal(got.cpu().numpy(), want(case, k, first, last))
    check_attn(case, *run_attn(case, c, page_idx=got), page_idx=got.cpu())


def raw_select(score_rows, k, first=0, last=0, seed=0):
    """Selection over prescribed scores: d = 64, one query row e_0 = 1, lo = hi = the score in channel 0."""
    score_rows = np.asarray(score_rows, np.float32)
    B, n = score_rows.shape
    dims = _lib.PagedDims(batch=B, new_len=1, n_heads_q=1, n_heads_kv=1, head_dim=64, dtype=PD_FP32, cache_dtype=PD_FP32,
                          page_rows=16, n_pages=B * n, max_pages=n, causal=1)
    q = torch.zeros(B, 1, 1, 64, device="cuda")
    q[..., 0] = 1
    bounds = torch.zeros(B * n, 1, 2, 64, device="cuda")
    bounds[:, 0, :, 0] = torch.from_numpy(score_rows).reshape(-1, 1).cuda()
    table = torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n)
    pages = torch.zeros(B * n, 1, 16, 64, device="cuda")
    cache = _lib.PagedCache(dims, pages, pages, table, torch.full((B,), n * 16, dtype=torch.int32, device="cuda"),
                            k_bounds=bounds)
    out = torch.empty(B, 1, k, dtype=torch.int32, device="cuda")
    ws = torch.empty(_lib.pd_paged_workspace_bytes(dims, k, 0), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_select(dims, cache, q, k, first, last, out, ws)
    return out[:, 0].cpu().numpy()


@pytest.mark.parametrize("n", [1, 2, 511, 512, 513, 2048, 2049, 4097, 8192, 9000])
def test_ties_and_special_scores(gpu_lib, n):
    """Equal scores (all, or in long runs), signed zeros, infinities and NaN, over one and several turns of the threads
    and beyond the registers."""
    rng = np.random.default_rng(n)
    rows = [np.zeros(n), rng.integers(-3, 4, n).astype(float), rng.standard_normal(n), np.where(rng.random(n) < 0.5, 0.0, -0.0),
            np.where(rng.random(n) < 0.3, -np.inf, rng.integers(0, 2, n)), np.where(rng.random(n) < 0.01, np.nan, rng.standard_normal(n)),
            np.where(rng.random(n) < 0.1, np.inf, rng.standard_normal(n)), np.arange(n) * 1e-7 + 1]
    rows = np.asarray(rows, np.float32)
    for k in sorted({1, min(3, n), min(64, n), n // 2 or 1, n}):
        for first, last in ((0, 0), (1, 2), (n, 0)):
            got = raw_select(rows, k, first, last)
            for r, row in enumerate(rows):
                assert got[r].tolist() == ref.select_ref(row.astype(np.float64), k, first, last), (n, k, first, last, r)


def test_near_ties_are_told_apart(gpu_lib):
    """Scores that differ by one unit in the last place of the sum's double: sums of products whose fp32 sum is equal."""
    d, n = 64, 64
    g = torch.Generator().manual_seed(3)
    case = Case([n * 16], hq=1, hkv=1, d=d, dtype=PD_BF16, R=16, seed=3)
    case.q[:] = torch.randn(1, 1, 1, d, generator=g).to(torch.bfloat16)
    base = torch.randn(d, generator=g).to(torch.bfloat16)
    for j in range(n):
        x = base.clone()
        x[j] = (x[j].float() * (1 + 2.0 ** -7)).to(torch.bfloat16)
        case.pool["bounds"][int(case.table[0, j]), 0, :] = x
    c = case.to_gpu()
    for k in (1, 7, 31, 63):
        assert np.array_equal(select(case, c, k, 0, 0).cpu().numpy(), want(case, k, 0, 0))


def test_page_lists_of_the_callers(gpu_lib):
    """Entries of -1 and beyond the table are skipped, pages behind the rows add nothing, a page named twice counts
    twice, an empty list gives zeros."""
    case = Case([100, 100], hq=2, hkv=1, d=64, R=16, seed=5, max_pages=8)
    c = case.to_gpu()
    idx = torch.tensor([[[3, -1, 0, 8, 7]], [[-1, -1, 1 << 30, -(1 << 31), 7]]], dtype=torch.int32)
    o, lse = run_attn(case, c, page_idx=idx.cuda())
    check_attn(case, o, lse, page_idx=idx)
    assert torch.all(o[1] == 0) and torch.all(lse[1] == -math.inf)
    one, l1 = run_attn(case, c, page_idx=torch.tensor([[[2, -1]], [[2, -1]]], dtype=torch.int32).cuda())
    two, l2 = run_attn(case, c, page_idx=torch.tensor([[[2, 2]], [[2, 2]]], dtype=torch.int32).cuda())
    np.testing.assert_allclose(h64(l2), h64(l1) + math.log(2), atol=1e-5)
    np.testing.assert_allclose(h64(two), h64(one), rtol=2.0 ** -7, atol=2.0 ** -7)


@pytest.mark.parametrize("dtype,cache", [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)], ids=["bf16", "fp8", "fp32"])
def test_the_bound_holds_for_the_keys_of_a_page(gpu_lib, dtype, cache):
    """Bounds and rows as pd_paged_append writes them.  No given key has a larger product with a query than its page's
    score; a key that the pages hold exceeds it by its rounding to E4M3 at most, and can (a key of 1.9375 is held as
    2, one of -1.9375 as -2)."""
    n, R, d = 150, 32, 64
    case = Case([n], new_len=n, hq=4, hkv=2, d=d, dtype=dtype, cache=cache, R=R, seed=11)
    case.k_rows[0][70:90] = 1.9375 * torch.sign(case.k_rows[0][70:90])
    c = case.to_gpu()
    k = case.k_rows[0][None].cuda()
    _lib.pd_paged_append(case.dims, c["cache"], k, k)
    held = [torch.empty(1, 2, n, d, dtype=case.q.dtype, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(case.dims, c["cache"], 0, n, *held)
    bounds, q, given, held = h64(c["bounds"]), h64(case.q[0]), h64(case.k_rows[0]), h64(held[0][0])
    beyond = 0
    for g in range(2):
        rows = q[:, 2 * g:2 * g + 2].reshape(-1, d)
        for j in range(-(-n // R)):
            lo, hi = bounds[int(case.table[0, j]), g]
            score = np.where(rows >= 0, rows * hi, rows * lo).sum(-1)[:, None]
            x, y = given[j * R:(j + 1) * R, g], held[g, j * R:(j + 1) * R]
            tiny = 1e-12 * (np.abs(rows) @ np.abs(x).T)                 # this test's own sums in double
            assert np.all(rows @ x.T <= score + tiny)
            off = np.abs(rows) @ (2.0 ** -4 * np.abs(x) + 2.0 ** -17 * np.abs(x).max(-1, keepdims=True) + 2.0 ** -110).T
            assert np.all(rows @ y.T <= score + tiny + (off if cache == PD_FP8_E4M3 else 0))
            beyond += int((rows @ y.T > score + tiny).sum())
    assert beyond == 0 or cache == PD_FP8_E4M3
    ones = np.ones(d)                                                   # one row of equal keys: its page's score is its product
    case = Case([1], hq=1, hkv=1, d=d, dtype=dtype, cache=cache, R=16, seed=1)
    c = case.to_gpu()
    k = torch.full((1, 1, 1, d), 1.9375, dtype=case.q.dtype, device="cuda")
    _lib.pd_paged_append(case.dims, c["cache"], k, k)
    held = [torch.empty(1, 1, 1, d, dtype=case.q.dtype, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(case.dims, c["cache"], 0, 1, *held)
    score = (ones * h64(c["bounds"])[int(case.table[0, 0]), 0, 1]).sum()
    assert score == 1.9375 * d and ones @ h64(held[0][0, 0, 0]) == (2.0 if cache == PD_FP8_E4M3 else 1.9375) * d
