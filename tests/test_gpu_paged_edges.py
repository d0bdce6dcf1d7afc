"""Where the paged attention's rows part: page ids outside the pool and values that are not finite, which count for the
rows that see them and for no others, wherever they lie."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged_case import HALF_STEP, Case, check_attn, h64, run_attn
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp32"]


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("hq,hkv,L,n,bad", [(4, 2, 24, 60, 3),      # 48 rows, two row blocks; the page holds new rows
                                            (3, 1, 33, 90, 4),      # 99 rows, four row blocks
                                            (4, 4, 7, 40, 2),       # one block; the page's rows are all new
                                            (8, 1, 40, 3000, 186),  # 320 rows, keys cut into parts
                                            (8, 1, 40, 3000, 2)])   # a page that every row sees
def test_a_bad_page_spoils_the_rows_that_see_it(gpu_lib, dtype, cache, hq, hkv, L, n, bad):
    """Causal rows: those whose own position lies before the page keep their attention, whatever block of rows they are
    taken in; without a causal mask all rows see it.  The other sequence is left alone."""
    R, d = 16, 64
    for causal in (1, 0):
        case = Case([n, n], new_len=L, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, R=R, causal=causal, seed=L)
        c = case.to_gpu()
        for number in (case.dims.n_pages, -3, (1 << 31) - 1):
            c["table"][1, bad] = number
            o, lse = run_attn(case, c)
            clean = min(L, max(0, bad * R - (n - L))) if causal else 0   # new rows before the page
            assert torch.isnan(o[1, clean:]).all() and torch.isnan(lse[1, :, clean:]).all()
            o[1, clean:], lse[1, :, clean:] = 7.0, 7.0
            part = Case.__new__(Case)
            part.__dict__.update(case.__dict__, lens=[n, n - L + clean], new=[L, clean])
            part.held = {k: [v[0], v[1][:n - L + clean]] for k, v in case.held.items()}
            check_attn(part, o, lse)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_a_bad_page_in_a_list(gpu_lib, dtype, cache):
    """Lists of pages: one that names the bad page is NaN for the rows that see it, one that does not is not."""
    R, n, L = 16, 64, 20
    case = Case([n], new_len=L, hq=4, hkv=2, d=64, dtype=dtype, cache=cache, R=R, seed=3)
    c = case.to_gpu()
    c["table"][0, 3] = case.dims.n_pages + 5                          # positions 48..63: new rows 4..19
    idx = torch.tensor([[[3, 0, 1], [0, 2, -1]]], dtype=torch.int32, device="cuda")
    o, lse = run_attn(case, c, page_idx=idx)
    assert torch.isnan(o[0, 4:, :2]).all() and torch.isnan(lse[0, :2, 4:]).all()
    assert torch.isfinite(o[0, :4, :2]).all() and torch.isfinite(o[0, :, 2:]).all() and torch.isfinite(lse[0, 2:]).all()
    part = Case.__new__(Case)
    part.__dict__.update(case.__dict__, lens=[n - L + 4], new=[4])
    part.held = {k: [v[0][:n - L + 4]] for k, v in case.held.items()}
    o[:, 4:], lse[:, :, 4:] = 7.0, 7.0
    check_attn(part, o, lse, page_idx=idx.cpu())


@pytest.mark.parametrize("dtype", [PD_BF16, PD_FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values_count_with_their_weight_wherever_they_lie(gpu_lib, dtype, d):
    """An infinite value whose weight is there gives its infinity; one whose weight has underflowed (e^-400 of the
    largest) gives 0 * inf = NaN: among whole steps, in the last keys of a single row, and at positions that some of
    several causal rows see.  Other channels and rows are finite, whatever the place."""
    n = 700
    for L, at in ((1, 40), (1, n - 1), (1, n - 20), (4, 40), (4, n - 4), (4, n - 3), (40, n - 38), (40, 300)):
        for score, top in ((400.0, 17), (400.0, at - 5), (0.0, 17)):  # of one key above all others, the infinite one's too
            for bad in (math.inf, -math.inf):
                case = Case([n], new_len=L, hq=2, hkv=2, d=d, dtype=dtype, R=32, seed=L)
                for x in (case.q, *case.k_rows):
                    x.zero_()
                case.q[:, :, :, 0] = 160.0 * math.sqrt(d / 64)        # score = q_0 k_0 / sqrt(d)
                case.k_rows[0][top, :, 0] = score / 20
                case.v_rows[0][at, 0, 5] = bad
                case.place()
                o, lse = run_attn(case, case.to_gpu())
                first = max(0, at - (n - L))                          # the first new row that sees it
                hit = o[0, first:, 0, 5].float()
                assert torch.isnan(hit).all() if score else (hit == bad).all(), (L, at, score, bad, hit)
                o[0, first:, 0, 5] = 0.0
                assert torch.isfinite(o).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_nan_values_spoil_their_channel_alone(gpu_lib, dtype, cache):
    """A NaN value, however small its weight, in whole and in masked steps.  In 8 bits too: the row's other channels
    keep their values."""
    n = 700
    for L, at in ((1, 40), (1, n - 1), (4, 40), (4, n - 3), (40, n - 38)):
        for score, top in ((400.0, 17), (400.0, at - 5), (0.0, 17)):
            case = Case([n], new_len=L, hq=2, hkv=2, d=64, dtype=dtype, cache=cache, R=32, seed=L)
            for x in (case.q, *case.k_rows):
                x.zero_()
            case.q[:, :, :, 0] = 160.0
            case.k_rows[0][top, :, 0] = score / 20
            case.v_rows[0][at, 0, 5] = math.nan
            case.place()
            o, lse = run_attn(case, case.to_gpu())
            first = max(0, at - (n - L))
            assert torch.isnan(o[0, first:, 0, 5]).all()
            o[0, first:, 0, 5] = 0.0
            assert torch.isfinite(o).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("cache", [PD_BF16, PD_FP8_E4M3], ids=["bf16", "fp8"])
@pytest.mark.parametrize("hq,hkv,L,lens,d", [(4, 4, 1, [3, 40, 300], 64), (28, 4, 1, [700, 33, 2], 128), (16, 1, 1, [5000, 129], 128),
                                             (4, 2, 8, [90, 2000], 64), (2, 2, 16, [16, 260], 128)])
def test_weights_of_sixteen_bits(gpu_lib, cache, hq, hkv, L, lens, d):
    """Up to 16 query rows a KV head the weights multiply V as two bf16 terms: the first cut off (the second is below
    2^-7 of the weight), the second rounded (2^-8 of itself): 2^-15 of the weight together.  The rest as in check_attn."""
    case = Case(lens, new_len=L, hq=hq, hkv=hkv, d=d, cache=cache, R=32, seed=hq + L)
    o, lse = run_attn(case, case.to_gpu())
    check_attn(case, o, lse)
    G = hq // hkv
    for b in range(len(lens)):
        for g in range(hkv):
            k, v = case.held["k"][b][:, g], case.held["v"][b][:, g]
            want, _, mass, spread = ref.attn_ref(case.rows_of(b, g), k, v, case.ends(b), case.scale)
            delta = (2 * (d + 4) * 2.0 ** -24 * spread + 2.0 ** -21 + len(k) * 2.0 ** -24)[:, None]
            err = np.abs(h64(o[b, :, g * G:(g + 1) * G]).reshape(-1, d) - want)
            assert np.all(err <= mass * (2 * delta + 2.0 ** -15) + np.abs(want) * HALF_STEP[PD_BF16] + 1e-37)


@pytest.mark.parametrize("dtype", [PD_BF16, PD_FP32])
def test_infinite_keys(gpu_lib, dtype):
    """A key with an infinite element: where the score is -inf the key is as if it were not there, where it is +inf the row
    is NaN (inf - inf).  In whole steps and at a new row's position, which the rows before do not see."""
    seen = []
    for L, n, at in ((6, 50, 47), (1, 700, 20), (6, 700, 20), (40, 700, 690)):
        for bad in (math.inf, -math.inf):
            case = Case([n], new_len=L, hq=8, hkv=2, d=128, dtype=dtype, R=16, seed=12)
            case.k_rows[0][at, 0, 3] = bad
            case.place()
            o, lse = run_attn(case, case.to_gpu())
            for g in range(2):
                keep = np.arange(n) != (at if g == 0 else n)
                q, k, v = case.rows_of(0, g), case.held["k"][0][keep, g], case.held["v"][0][keep, g]
                want, l, mass, spread = ref.attn_ref(q, k, v, case.ends(0), case.scale, np.arange(n)[keep])
                delta = (2 * (128 + 4) * 2.0 ** -24 * spread + 2.0 ** -21 + n * 2.0 ** -24)[:, None]
                tol = mass * (2 * delta + (2.0 ** -8 if dtype == PD_BF16 else 0)) + np.abs(want) * HALF_STEP[dtype] + 1e-37
                got, gl = h64(o[0, :, 4 * g:4 * g + 4]).reshape(-1, 128), h64(lse[0, 4 * g:4 * g + 4]).T.reshape(-1)
                above = (case.ends(0) > at) & (q[:, 3] * bad > 0) & (g == 0)
                seen += [above.sum(), ((case.ends(0) > at) & ~above).sum()] if g == 0 else []
                assert np.all(np.isnan(got[above])) and np.all(np.isnan(gl[above]))
                rest = ~above
                assert np.all(np.abs(got - want)[rest] <= tol[rest])
                assert np.all(np.abs(gl - l)[rest] <= (delta[:, 0] + 2.0 ** -21 * (1 + np.abs(l)))[rest])
    assert sum(seen[::2]) > 20 and sum(seen[1::2]) > 20               # rows with scores of +inf, and of -inf
