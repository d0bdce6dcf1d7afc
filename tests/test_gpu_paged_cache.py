"""pd_paged_append and pd_paged_read: every bit of the pool, written or not, against the oracle; read-back; the prefix
of a compact decode."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged_case import TORCH, Case, h64
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)]


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def append_all(case, c, steps, stride_extra=0):
    """Appends the rows of every sequence in `steps` calls of new_len rows each, the last one first short."""
    d = case.dims
    L, done = d.new_len, [0] * d.batch
    for s in range(steps):
        new = [min(L, n - at) for n, at in zip(case.lens, done)]
        fused = torch.full((d.batch, L, 2 * d.n_heads_kv + stride_extra, d.head_dim), math.nan, dtype=TORCH[d.dtype])
        for b in range(d.batch):
            fused[b, :new[b], :d.n_heads_kv] = case.k_rows[b][done[b]:done[b] + new[b]]
            fused[b, :new[b], d.n_heads_kv:2 * d.n_heads_kv] = case.v_rows[b][done[b]:done[b] + new[b]]
            done[b] += new[b]
        fused = fused.cuda()
        c["kv_len"].copy_(torch.tensor(done, dtype=torch.int32))
        c["new_rows"].copy_(torch.tensor(new, dtype=torch.int32))
        _lib.pd_paged_append(d, c["cache"], fused[:, :, :d.n_heads_kv], fused[:, :, d.n_heads_kv:2 * d.n_heads_kv])
    assert done == case.lens


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("R,L,lens,d,hkv", [(16, 1, [1, 3, 17, 0], 64, 2), (16, 33, [33, 5, 64, 0, 47], 128, 1),
                                            (64, 70, [131, 64, 1], 128, 3), (256, 300, [300, 256, 511], 64, 2),
                                            (32, 7, [40, 32, 31], 128, 4)])
def test_append_writes_every_row_and_nothing_else(gpu_lib, dtype, cache, R, L, lens, d, hkv):
    print(f"[append] {dtype}/{cache} R={R} L={L} lens={lens}", flush=True)
    case = Case(lens, new_len=L, hq=hkv, hkv=hkv, d=d, dtype=dtype, cache=cache, R=R, seed=R + L)
    want = {k: v.clone() for k, v in case.pool.items() if v is not None}
    for name in ("k", "v"):                        # an empty pool: marks everywhere
        case.pool[name] = torch.full_like(case.pool[name], 0x7F if case.fp8 else math.nan)
    case.pool["bounds"] = torch.full_like(case.pool["bounds"], math.nan)
    if case.fp8:
        for name in ("k_exp", "v_exp"):
            case.pool[name] = torch.full_like(case.pool[name], 255)
    c = case.to_gpu()
    append_all(case, c, max(-(-n // L) for n in lens), stride_extra=1)
    for name in want:
        assert torch.equal(bits(c[name].cpu()), bits(want[name])), name


def test_append_of_special_values(gpu_lib):
    """Rows of zeros, of one value at every power of two, subnormal, huge, with NaN and infinities: the 8-bit rows of
    the oracle bit for bit (NaN as NaN)."""
    case = Case([120], new_len=120, hq=1, hkv=1, d=64, cache=PD_FP8_E4M3, R=64, seed=3)
    x = case.k_rows[0]
    for i in range(60):
        x[i] *= 2.0 ** (4 * i - 120)
    x[60] = 0
    x[61] = -0.0
    x[62, 0, :] = 448.0
    x[63, 0, :] = torch.linspace(-448, 448, 64).to(x.dtype)
    x[64, 0, 3] = math.inf
    x[65, 0, 4] = -math.inf
    x[66, 0, 5] = math.nan
    x[67] = math.nan
    x[68] = 3.3e38
    x[69] = torch.finfo(torch.bfloat16).max
    x[70] = 1e-40
    c = case.to_gpu()
    k = x[None].cuda()
    _lib.pd_paged_append(case.dims, c["cache"], k, k)
    val, e = ref.quantise_ref(h64(x))
    got, ge = (torch.cat([c[n][int(case.table[0, j])] for j in range(2)], 1)[:, :120].cpu() for n in ("k", "k_exp"))
    assert np.array_equal(ge.numpy()[0].astype(int) - 127, e[:, 0])
    np.testing.assert_array_equal(got[0].view(torch.float8_e4m3fn).double().numpy(), val[:, 0])


@pytest.mark.parametrize("dtype", [PD_BF16, PD_FP32])
def test_bounds(gpu_lib, dtype):
    """A page begins anew with its row 0, is widened otherwise; a row written twice keeps the wider bounds; NaNs do not
    count."""
    case = Case([20], new_len=20, hq=1, hkv=1, d=64, dtype=dtype, R=16, seed=4)
    c = case.to_gpu()
    x = case.k_rows[0].clone()
    x[3, 0, 7] = math.nan
    _lib.pd_paged_append(case.dims, c["cache"], x[None].cuda(), x[None].cuda())
    p0, p1 = (int(case.table[0, j]) for j in range(2))
    y = x.float()
    lo = torch.where(torch.isnan(y), math.inf, y)
    hi = torch.where(torch.isnan(y), -math.inf, y)
    got = c["bounds"].cpu().float()
    assert torch.equal(got[p0, 0, 0], lo[:16, 0].amin(0)) and torch.equal(got[p0, 0, 1], hi[:16, 0].amax(0))
    assert torch.equal(got[p1, 0, 0], lo[16:, 0].amin(0)) and torch.equal(got[p1, 0, 1], hi[16:, 0].amax(0))
    # Position 19 again, with another row: page 1 is widened, page 0 stays.
    d1 = _lib.PagedDims.from_buffer_copy(case.dims)
    d1.new_len = 1
    c["new_rows"].fill_(1)
    z = (torch.randn(1, 1, 1, 64) * 3).to(x.dtype)
    _lib.pd_paged_append(d1, c["cache"], z.cuda(), z.cuda())
    new = c["bounds"].cpu().float()
    assert torch.equal(new[p0], got[p0])
    assert torch.equal(new[p1, 0, 0], torch.minimum(got[p1, 0, 0], z[0, 0, 0].float()))
    assert torch.equal(new[p1, 0, 1], torch.maximum(got[p1, 0, 1], z[0, 0, 0].float()))


def test_append_out_of_place_values(gpu_lib):
    """More new rows than the sequence holds, lengths beyond the table, negative ones, page ids outside the pool: what
    cannot be placed is not written, the rest is."""
    case = Case([16, 16, 16, 16], new_len=8, hq=1, hkv=1, d=64, R=16, seed=5)
    c = case.to_gpu()
    before = c["k"].clone()
    c["table"][1, 0] = case.dims.n_pages
    c["table"][2, 0] = -1
    c["kv_len"].copy_(torch.tensor([5, 8, 8, -3], dtype=torch.int32))
    c["new_rows"].copy_(torch.tensor([8, 8, 8, 8], dtype=torch.int32))
    x = torch.randn(4, 8, 1, 64).to(torch.bfloat16).cuda()
    _lib.pd_paged_append(case.dims, c["cache"], x, x)
    p = int(case.table[0, 0])
    want = before.clone()
    want[p, 0, :5] = x[0, 3:, 0]                   # rows 0..2 would lie before position 0
    assert torch.equal(bits(c["k"]), bits(want))
    # A length beyond the table counts as the table's.
    c["kv_len"].copy_(torch.tensor([1000, 0, 0, 0], dtype=torch.int32))
    _lib.pd_paged_append(case.dims, c["cache"], x, x)
    want[p, 0, 8:] = x[0, :, 0]
    assert torch.equal(bits(c["k"]), bits(want))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("R,d,lens,first,n", [(16, 64, [37, 1, 0, 64], 0, 64), (64, 128, [200, 129], 63, 70),
                                              (256, 128, [300], 299, 1), (32, 64, [95, 96, 97], 31, 66)])
def test_read_back(gpu_lib, dtype, cache, R, d, lens, first, n):
    case = Case(lens, hq=3, hkv=3, d=d, dtype=dtype, cache=cache, R=R, seed=n)
    c = case.to_gpu()
    ko, vo = (torch.full((len(lens), 3, n, d), 5.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    _lib.pd_paged_read(case.dims, c["cache"], first, n, ko, vo)
    for name, out in (("k", ko), ("v", vo)):
        for b in range(len(lens)):
            m = max(0, min(lens[b] - first, n))
            # E4M3 times a power of two has four significant bits: exact in bf16
            assert np.array_equal(h64(out[b, :, :m]), case.held[name][b][first:first + m].transpose(1, 0, 2))
            assert torch.all(out[b, :, m:] == 5.0)


def test_read_back_of_a_bad_page_is_nan(gpu_lib):
    for dtype, cache in KINDS:
        case = Case([40, 40], hq=1, hkv=1, d=64, dtype=dtype, cache=cache, R=16, seed=9)
        c = case.to_gpu()
        c["table"][0, 1] = 1 << 30
        ko, vo = (torch.full((2, 1, 40, 64), 5.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
        _lib.pd_paged_read(case.dims, c["cache"], 0, 40, ko, vo)
        for out in (ko, vo):
            assert torch.isnan(out[0, 0, 16:32]).all() and torch.isfinite(out[0, 0, :16]).all()
            assert torch.isfinite(out[0, 0, 32:]).all() and torch.isfinite(out[1]).all()
