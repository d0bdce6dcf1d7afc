"""pd_paged_window_attn at the sizes of many rows: softmax scales next to the least that the kernel of many rows takes, and
rows in fp32, which it does not take."""

import pytest
import torch

from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP4_E2M1, PD_FP8_E4M3
from test_gpu_paged_window import check, hide, make, run, run_window

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_FP4_E2M1)]


@pytest.mark.parametrize("kind", KINDS, ids=["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("scale", [2e-30, 1.0000001e-30, 1e-30, 0.9999e-30, 1e-37, 1e-41, 1.4e-45])
def test_scales_that_vanish(gpu_lib, kind, causal, scale):
    """All visible keys weigh the same, masked ones nothing, whichever kernel runs."""
    case = make(kind, [70, 200, 0, 33], new_len=33, new=[33, 33, 0, 20], hq=64, hkv=64, d=64, R=16, causal=causal, seed=3, sm_scale=scale)
    c = case.to_gpu()
    hide(case, c, 40, 3)
    o, lse = run_window(case, c, 40, 3)
    check(case, o, lse, 40, 3)


def test_the_scale_chooses_the_kernel(gpu_lib):
    """The kernel of many rows needs no workspace; the other one, which takes scales that vanish, cuts long windows."""
    dims = make(KINDS[0], [100], new_len=33, hq=9, hkv=9, d=64, R=16).dims
    dims.batch, dims.max_pages = 16, 1000
    size = lambda scale: _lib.pd_paged_window_workspace_bytes(_with(dims, scale), 9000, 0)  # noqa: E731
    assert size(0.0) == size(1.0) == size(1e-29) == 0 and size(0.9e-30) == size(1e-45) > 0


def _with(dims, scale):
    d = _lib.PagedDims.from_buffer_copy(dims)
    d.sm_scale = scale
    return d


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,hq,hkv,d,new", [(33, 32, 32, 64, [33, 33, 5, 0, 33]), (70, 32, 8, 128, [70, 1, 70, 64, 69])])
def test_many_rows_in_fp32(gpu_lib, causal, L, hq, hkv, d, new):
    """More blocks of 32 rows than CUs."""
    lens = [n + m for n, m in zip(new, (0, 211, 40, 7, 100))]
    for window, sinks in ((50, 3), (1 << 30, 0)):
        run("fp32", (PD_FP32, PD_FP32), lens, window, sinks, new_len=L, new=new, hq=hq, hkv=hkv, d=d, R=16, causal=causal, seed=L)
