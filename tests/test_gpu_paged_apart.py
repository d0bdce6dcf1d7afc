"""What a query row of the paged attention does not see leaves every bit of its output as it is, also where it changes what
other rows of the same workgroup get."""

import math

import numpy as np
import pytest
import torch

from paged_case import run_attn
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP4_E2M1, PD_FP8_E4M3
from test_gpu_paged_window import make, run_window

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_FP4_E2M1), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp4", "fp32"]


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("window", [False, True])
@pytest.mark.parametrize("L,hq,hkv,d", [(3, 8, 2, 64), (12, 8, 2, 64), (5, 3, 1, 128), (40, 2, 1, 128)])
def test_a_key_that_others_see(gpu_lib, kind, window, L, hq, hkv, d):
    """A key as it is, much larger, of NaN and of infinities, in a late step of the wave that takes it: the rows that do not
    see it keep their bits, whichever of these makes the others' running maximum jump."""
    blocks = 4                                              # of 128 keys, in fp32 64: the keys of a unit are not cut
    keys = blocks * (64 if kind[0] == PD_FP32 else 128)
    n, W = keys - 9, keys - 100
    for at in (n - 2, n - L + 1) + ((n - W - 1,) if window else ()):
        got = []
        for change in ("none", "large", "nan", "inf", "-inf"):
            if "inf" in change and kind[1] in (PD_FP8_E4M3, PD_FP4_E2M1):
                continue
            case = make(kind, [n + (700 if window else 0)], new_len=L, hq=hq, hkv=hkv, d=d, R=16, seed=L)
            p = at + (700 if window else 0)
            if change == "large":
                case.k_rows[0][p] *= 60
            elif change != "none":
                case.k_rows[0][p, :, 3] = float(change)
            case.place()
            c = case.to_gpu()
            got.append((change, *(run_window(case, c, W, 2) if window else run_attn(case, c))))
        own = np.arange(n - L, n)
        sees = (at <= own) & (at > own - (W if window else n))
        far = torch.from_numpy(np.flatnonzero(~sees))
        assert len(far) > 0 and sees.any()
        for change, o, lse in got[1:]:
            assert torch.equal(o[:, far], got[0][1][:, far]), (at, change)
            assert torch.equal(lse[:, :, far], got[0][2][:, :, far]), (at, change)
            assert change == "none" or not torch.equal(o, got[0][1]), (at, change)


@pytest.mark.parametrize("window", [False, True])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,hq,hkv,d", [(6, 8, 2, 64), (6, 8, 2, 128), (3, 2, 2, 128), (70, 1, 1, 64), (70, 88, 88, 64)])
def test_values_that_4_bits_read_as_infinite(gpu_lib, window, causal, L, hq, hkv, d):
    """A value from 1.75 * 2^127 on is held as 4 * 2^126, which reads as infinity: the rows that do not see it keep their
    bits, the others get the infinity in its channel, and numbers in the others."""
    n, W = 100, 20
    kind = (PD_BF16, PD_FP4_E2M1)
    for at in (n - 1, n - L // 2, max(n - L - 15, 10)):
        clean = make(kind, [n], new_len=L, hq=hq, hkv=hkv, d=d, R=16, causal=causal, seed=L)
        call = lambda case: run_window(case, case.to_gpu(), W, 2) if window else run_attn(case, case.to_gpu())  # noqa: E731
        was, lse = call(clean)
        for sign, value in ((1, 3.3e38), (-1, 3.3e38), (1, 1.75 * 2.0 ** 127), (-1, 1.625 * 2.0 ** 127)):
            case = make(kind, [n], new_len=L, hq=hq, hkv=hkv, d=d, R=16, causal=causal, seed=L)
            ch = d - 5
            case.v_rows[0][at, 0, ch] = sign * value
            case.place()
            o, l = call(case)
            own = np.arange(n - L, n)
            sees = ((at <= own) if causal else (own < n)) & (at > own - (W if window else n))
            far, near = (torch.from_numpy(np.flatnonzero(x)) for x in (~sees, sees))
            G = hq // hkv
            assert torch.equal(l, lse)
            assert torch.equal(o[:, far], was[:, far]) and torch.equal(o[:, :, G:], was[:, :, G:]), (at, value)
            hit = o[0, near, :G].float().cpu()
            if value >= 1.75 * 2.0 ** 127:                  # below, 256 * |v| may pass 2^128
                assert torch.all(hit[..., ch] == sign * math.inf), (at, value)
            rest = torch.ones(d, dtype=torch.bool)
            rest[ch // 32 * 32:] = False
            assert torch.equal(hit[..., rest], was[0, near, :G].float().cpu()[..., rest])
            assert torch.isfinite(torch.cat([hit[..., :ch], hit[..., ch + 1:]], -1)).all()
