"""pd_paged_window_attn where the new rows of a KV head are many and so are the row blocks: keys in tiles, 64 or 128 query
rows a workgroup.  Against float64, over a pool that holds NaN wherever no row lies."""

import math

import numpy as np
import pytest
import torch

from paged_case import h64
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP4_E2M1, PD_FP8_E4M3
from test_gpu_paged_window import check, hide, make, run, run_window  # noqa: F401

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_FP4_E2M1)]
IDS = ["bf16", "fp8", "fp4"]


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,hq,hkv,d,R", [(64, 32, 32, 64, 16), (33, 32, 16, 128, 64), (130, 16, 8, 64, 32), (20, 84, 12, 128, 256),
                                          (257, 8, 8, 128, 16)])
def test_windows_and_first_positions(gpu_lib, kind, causal, L, hq, hkv, d, R):
    """Windows of one position, across a tile, across several and wider than the sequences; sequences of nothing but new
    rows, of few of them, without any."""
    for i, (window, sinks) in enumerate([(1, 0), (37, 3), (100, 70), (1 << 30, 5)][L % 2::2]):
        lens = [L, 600 + 13 * i, 3 * L + 5, L + 1, 311 + L, 0, 500, L + 64]
        new = [L, L, L - 1, 1, L, 0, L // 2, L]
        run("tile", kind, lens, window, sinks, new_len=L, new=new, hq=hq, hkv=hkv, d=d, R=R, causal=causal, seed=i + L)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_128_rows_a_workgroup(gpu_lib, kind):
    g = torch.Generator().manual_seed(1)
    B, L = 8, 60
    lens = [int(x) for x in torch.randint(0, 400, (B,), generator=g)]
    new = [min(L, n, int(x)) for n, x in zip(lens, torch.randint(0, 90, (B,), generator=g))]
    for causal in (0, 1):
        for d in (64, 128):
            run("128", kind, lens, 90, 4, new_len=L, new=new, hq=64, hkv=16, d=d, R=16, causal=causal, seed=d)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("B,L,hq,hkv,d,R", [(5, 33, 28, 28, 64, 16), (3, 9, 180, 45, 128, 16), (1, 260, 32, 8, 128, 64), (1, 449, 16, 4, 64, 128),
                                            (4, 48, 136, 136, 64, 32)])
def test_blocks_around_the_least_that_fill_the_card(gpu_lib, kind, B, L, hq, hkv, d, R):
    """Blocks of 32 rows just above 256, and below: fewer than 64 rows a KV head, many."""
    lens = [900, 5, L + 13, 0, 333][:B]
    for causal, window in ((1, 70), (0, 600)):
        run("around", kind, lens, window, 3, new_len=L, new=[L, min(5, L), L - 1, 0, L][:B], hq=hq, hkv=hkv, d=d, R=R, causal=causal, seed=L)


@pytest.mark.parametrize("hq,hkv,L", [(24, 24, 257), (12, 12, 530), (32, 8, 128), (39, 13, 100), (4, 2, 520)])
def test_padded_batches(gpu_lib, hq, hkv, L):
    """Most sequences with one new row or none: the row blocks that hold rows lie far apart, in runs of odd and even length."""
    B = 16
    new = [(L, 1, 1, 0, 2, 1, 70, 1)[i % 8] for i in range(B)]
    lens = [n + (0, 40, 211, 7, 500)[i % 5] for i, n in enumerate(new)]
    run("padded", KINDS[L % 3], lens, 90, 3, new_len=L, new=new, hq=hq, hkv=hkv, d=64, R=16, causal=L % 2, seed=L)


def test_more_than_sixteen_tiles(gpu_lib):
    """Windows of more than 1024 positions: where their groups lie is looked up again."""
    for window, sinks in ((2500, 130), (1 << 30, 0)):
        run("long", KINDS[0], [3000, 1100, 2049, 90], window, sinks, new_len=64, hq=64, hkv=64, d=64, R=64, new=[64, 9, 30, 64], seed=3)


def test_the_same_bits_again_and_no_workspace(gpu_lib):
    case, c, o, lse = run("again", KINDS[0], [700, 300, 500, 400], 200, 4, new_len=70, hq=64, hkv=32, d=128, R=16, seed=4)
    assert _lib.pd_paged_window_workspace_bytes(case.dims, 200, 4) == 0
    again = run_window(case, c, 200, 4)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    o2, _ = run_window(case, c, 200, 4, lse=False)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("d", [64, 128])
def test_nonfinite_rows_stay_with_the_rows_that_see_them(gpu_lib, kind, causal, which, d):
    """A NaN or an infinity at a position: the rows that do not see it keep their bits; the others get what the formula
    gives, also where all rows of a tile see it."""
    check_nonfinite(kind, causal, which, d, 70, 128)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("L,hkv", [(40, 136), (70, 256)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_nonfinite_rows_in_blocks_of_64_and_of_128(gpu_lib, kind, which, L, hkv):
    check_nonfinite(kind, 1, which, 64, L, hkv)


def check_nonfinite(kind, causal, which, d, L, hkv):
    W, n = 30, 200
    for bad in ((math.nan,) if kind[1] != PD_BF16 else (math.nan, math.inf, -math.inf)):
        for at in (1, 120, 150, 199):
            case = make(kind, [n], new_len=L, hq=hkv, hkv=hkv, d=d, R=16, causal=causal, seed=12)
            clean, _ = run_window(case, case.to_gpu(), W, 2)
            if at == 1 and (bad != bad) and which == "k":
                check(case, clean, None, W, 2)
            rows = case.k_rows if which == "k" else case.v_rows
            ch = d - 5
            rows[0][at, 0, ch] = bad
            case.place()
            o, _ = run_window(case, case.to_gpu(), W, 2)
            own = np.arange(n - L, n)
            sees = ((at <= own) if causal else (at < n)) & ((at > own - W) | (at < 2))
            far = torch.from_numpy(np.flatnonzero(~sees))
            assert torch.equal(o[:, far], clean[:, far]) and torch.equal(o[:, :, 1:], clean[:, :, 1:])
            near = torch.from_numpy(np.flatnonzero(sees))
            hit, was = o[0, near, 0].float().cpu(), clean[0, near, 0].float().cpu()
            if which == "v":
                x = hit[..., ch]
                assert torch.isnan(x).all() if math.isnan(bad) else torch.all(x == bad)
                keep = torch.ones(d, dtype=torch.bool)
                keep[ch] = False
                if kind[1] == PD_FP4_E2M1:
                    keep[ch // 32 * 32:ch // 32 * 32 + 32] = False
                if kind[1] != PD_FP8_E4M3:                            # another maximum scales the row's other values
                    assert torch.equal(hit[:, keep], was[:, keep])
            elif math.isnan(bad):
                assert torch.isnan(hit).all()


def test_values_of_several_kinds_in_many_tiles(gpu_lib):
    """Infinities of both signs and NaN in several tiles, at first positions and new rows: every row against the formula."""
    n, L, W, hkv = 400, 64, 150, 64
    case = make(KINDS[0], [n, L, L, L], new_len=L, hq=hkv, hkv=hkv, d=64, R=16, seed=5)
    for at, ch, v in ((0, 1, math.inf), (200, 2, math.nan), (260, 3, -math.inf), (300, 4, math.inf), (330, 4, -math.inf),
                      (370, 5, math.inf), (399, 63, math.nan)):
        case.v_rows[0][at, 7, ch] = v
    case.place()
    o, _ = run_window(case, case.to_gpu(), W, 1)
    o = h64(o)[0, :, 7]
    for r in range(L):
        p = n - L + r
        seen = [j for j in range(n) if j <= p and (j > p - W or j < 1)]
        v = case.held["v"][0][seen, 7]
        for ch in (1, 2, 3, 4, 5, 63):
            x = v[:, ch]
            special = x[~np.isfinite(x)]
            want = None if not len(special) else math.nan if np.isnan(special).any() or len(set(special)) > 1 else special[0]
            got = o[r, ch]
            assert np.isfinite(got) if want is None else (math.isnan(got) if math.isnan(want) else got == want), (r, ch, got, want)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_bad_pages_and_hidden_ones(gpu_lib, kind):
    """A page id outside the pool makes the rows NaN that see one of its positions, and no others."""
    L, W = 64, 10
    case = make(kind, [100, 164, 300, 64], new_len=L, hq=64, hkv=64, d=64, R=16, seed=3)
    c = case.to_gpu()
    hide(case, c, W, 3)
    good, gl = run_window(case, c, W, 3)
    check(case, good, gl, W, 3)
    for page in (case.dims.n_pages, -5):
        c["table"][1, 8] = page                       # positions 128..143; row r is position 100 + r
        o, lse = run_window(case, c, W, 3)
        hit = [r for r in range(L) if 100 + r >= 128 and 100 + r - W + 1 <= 143]
        rest = [r for r in range(L) if r not in hit]
        assert torch.equal(o[[0, 2, 3]], good[[0, 2, 3]]) and torch.equal(o[1, rest], good[1, rest])
        assert torch.isnan(o[1, hit]).all() and torch.isnan(lse[1, :, hit]).all() and torch.equal(lse[1, :, rest], gl[1, :, rest])
        c["table"][1, 8] = case.table[1, 8].item()


@pytest.mark.parametrize("causal", [0, 1])
def test_more_new_rows_than_positions(gpu_lib, causal):
    case = make(KINDS[0], [3, 0, 200, 70], new_len=70, new=[70, 70, 70, 70], hq=32, hkv=32, d=64, R=16, causal=causal, seed=4)
    for window, sinks in ((20, 1), ((1 << 31) - 1, (1 << 31) - 1)):
        o, lse = run_window(case, case.to_gpu(), window, sinks)
        check(case, o, lse, window, sinks)
        assert torch.all(o[1] == 0) and torch.all(lse[1] == -math.inf)


def test_scores_of_minus_infinity_and_large_ones(gpu_lib):
    case = make(KINDS[0], [300], new_len=64, hq=256, hkv=256, d=64, R=16, seed=6, sigma=3.0)
    case.k_rows[0][150:280, 5, 0] = -math.inf
    case.q[:, :, 5, 0] = 1.0
    case.place()
    o, lse = run_window(case, case.to_gpu(), 100, 0)
    own = np.arange(236, 300)
    for r, p in enumerate(own):
        seen = [j for j in range(p - 99, p + 1) if not 150 <= j < 280]
        if not seen:
            assert torch.all(o[0, r, 5] == 0) and float(lse[0, 5, r]) == -math.inf
        else:
            assert torch.isfinite(o[0, r, 5].float()).all() and math.isfinite(float(lse[0, 5, r]))
    case.k_rows[0][150:280, 5, 0] = 1.0
    case.place()
    check(case, *run_window(case, case.to_gpu(), 100, 0), 100, 0)
