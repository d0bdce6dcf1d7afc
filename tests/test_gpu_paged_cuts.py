"""Where the paged attention's keys are cut: walks of more than one window of 64 steps, batches of several groups of 64
sequences with and without a plan of their own, units of one size just below two a CU, lists of pages in large batches.
All sequences of a batch read the first kv_len rows of the same pages."""

import numpy as np
import pytest
import torch

from paged_case import Case, check_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp32"]
CUS = 256


def block_keys(dtype):
    """Keys that a workgroup takes at a time: four waves' steps of 32 keys (fp32: 16); a window is 64 such blocks."""
    return 64 if dtype == PD_FP32 else 128


class Batch:
    """lens[b] rows and new[b] new rows of sequence b, over the pages of one sequence; `run`, then `check` some."""

    def __init__(self, lens, L=1, new=None, seed=0, **kw):
        self.lens, self.new, B = list(lens), list(new or [L] * len(lens)), len(lens)
        self.case = Case([max(lens)], new_len=L, seed=seed, **kw)
        c = self.case.to_gpu()
        d = self.dims = _lib.PagedDims.from_buffer_copy(self.case.dims)
        d.batch = B
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn(B, L, d.n_heads_q, d.head_dim, generator=g).to(self.case.q.dtype)
        number = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.tensors = (c["k"], c["v"], c["table"].expand(B, -1).contiguous(), number(self.lens), number(self.new))
        self.cache = _lib.PagedCache(d, *self.tensors, c["k_exp"], c["v_exp"])

    def run(self, idx=None):
        d = self.dims
        o = torch.full_like(self.q, 7.0, device="cuda")
        lse = torch.full((d.batch, d.n_heads_q, d.new_len), 7.0, device="cuda")
        n = _lib.pd_paged_workspace_bytes(d, 0 if idx is None else idx.shape[-1], 1)
        assert n > 0                                                   # some keys may be cut: the walk is made
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        _lib.pd_paged_attn(d, self.cache, self.q.cuda(), o, lse, page_idx=None if idx is None else idx.cuda(), workspace=ws)
        torch.cuda.synchronize()
        return o, lse

    def check(self, o, lse, some, idx=None):
        for b in some:
            one = Case.__new__(Case)
            one.__dict__.update(self.case.__dict__, lens=[self.lens[b]], new=[self.new[b]], q=self.q[b:b + 1])
            one.held = {n: [x[0][:self.lens[b]]] for n, x in self.case.held.items()}
            check_attn(one, o[b:b + 1], lse[b:b + 1], page_idx=None if idx is None else idx[b:b + 1])


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("hq,L", [(2, 1), (3, 7)])
def test_walks_of_three_windows(gpu_lib, dtype, cache, hq, L):
    """As many equal units as CUs are not cut: every wave walks all blocks of its sequence, 130 of them, so that the window
    of pages and positions is filled three times by the loop of whole steps.  With a list of pages that begins
    with the last, partly filled one, and with one in descending order, the loop with masks walks them."""
    bk = block_keys(dtype)
    n, R, B = 129 * bk + 40, 64, CUS
    blocks = -(-n // bk)
    assert -(-B * blocks // CUS) == blocks > 2 * 64                    # the quota of an even batch: one part a unit
    batch = Batch([n] * B, L, hq=hq, hkv=1, d=64, dtype=dtype, cache=cache, R=R, seed=hq)
    batch.check(*batch.run(), (0, 101, B - 1))
    pages = -(-n // R)
    assert n % R and pages * R // bk > 2 * 64
    first_last = torch.tensor([pages - 1, *range(pages - 1)], dtype=torch.int32)
    for order in (first_last, torch.arange(pages - 1, -1, -1, dtype=torch.int32)):
        idx = order.expand(B, 1, pages).contiguous()
        batch.check(*batch.run(idx), (0, 101, B - 1), idx)


@pytest.mark.parametrize("B", [65, 127, 128, 129])
@pytest.mark.parametrize("kind", range(len(KINDS)), ids=IDS)
def test_cut_batches_of_two_groups(gpu_lib, B, kind):
    """Ragged batches of more than 64 sequences, which each wave walks by itself up to 128 of them and finds planned
    beyond: long sequences in the first group, at its border and in the second, empty ones and ones without new rows; 6, 36
    and 3 query rows a KV head (one and two row blocks)."""
    dtype, cache = KINDS[kind]
    g = torch.Generator().manual_seed(B + kind)
    hq, hkv = ((4, 2), (12, 1), (3, 3))[kind]
    for long in ((3,), (63, 64), (B - 1,), (0, 64, B - 1)):
        lens = torch.randint(0, 400, (B,), generator=g).tolist()
        new = torch.randint(0, 4, (B,), generator=g).tolist()
        for i, b in enumerate(long):
            lens[b], new[b] = 5000 - 700 * i, 3
        lens[1], new[2], lens[B - 2] = 0, 0, 1
        batch = Batch(lens, 3, new, hq=hq, hkv=hkv, d=64, dtype=dtype, cache=cache, R=16, seed=B)
        batch.check(*batch.run(), range(B))


@pytest.mark.parametrize("B,hkv", [(480, 1), (120, 4), (256, 2), (231, 2), (77, 6)])
@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_units_of_one_size_just_below_two_a_cu(gpu_lib, dtype, cache, B, hkv):
    """461 to 512 units whose keys are nearly as many: one whole part each, though tables and lengths would allow cuts.
    Planned by a launch (more than 128 sequences) and by the waves."""
    bk = block_keys(dtype)
    assert 1.8 * CUS <= B * hkv <= 2 * CUS
    lens = [21 * bk - 7 * (b % 50) for b in range(B)]
    blocks = [-(-n // bk) for n in lens]
    assert 0.8 * max(blocks) * B <= sum(blocks) and -(-sum(blocks) * hkv // CUS) >= max(blocks) > 16
    batch = Batch(lens, hq=2 * hkv, hkv=hkv, d=64, dtype=dtype, cache=cache, R=32, seed=B)
    batch.check(*batch.run(), (0, 49, B // 2, B - 1))


@pytest.mark.parametrize("B", [100, 130, 300])
@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_lists_of_pages_in_large_batches(gpu_lib, dtype, cache, B):
    """Lists of 1300 to 2600 keys that are cut, in batches with and without a plan: in any order, with absent entries and pages
    behind a sequence's end, over sequences of all lengths."""
    R, top_k, hkv = 64, 41, 2
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(1, 4000, (B,), generator=g).tolist()
    lens[0], lens[B // 2], lens[B - 1] = 4000, 0, 3999
    batch = Batch(lens, 2, [2 - b % 3 // 2 for b in range(B)], hq=6, hkv=hkv, d=64, dtype=dtype, cache=cache, R=R, seed=B)
    width = batch.dims.max_pages
    idx = torch.stack([torch.randperm(width, generator=g)[:top_k] for _ in range(B * hkv)]).to(torch.int32).view(B, hkv, top_k)
    idx[torch.rand(idx.shape, generator=g) < 0.2] = -1
    idx[1] = -1
    batch.check(*batch.run(idx), [0, 1, 2, 63, 64, 65, B // 2, B - 2, B - 1], idx)
