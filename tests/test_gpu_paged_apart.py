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
