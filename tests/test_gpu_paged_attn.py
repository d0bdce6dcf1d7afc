"""pd_paged_attn against float64, over a pool that holds NaN wherever no row lies."""

import math

import numpy as np
import pytest
import torch

from paged_case import Case, check_attn, h64, run_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp32"]


def run(name, *a, **kw):
    print(f"[attn] {name} {a} {kw}", flush=True)
    case = Case(*a, **kw)
    c = case.to_gpu()
    o, lse = run_attn(case, c)
    torch.cuda.synchronize()
    check_attn(case, o, lse)
    return case, c, o, lse


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (7, 1), (16, 2), (28, 4), (34, 2)])
def test_single_tokens(gpu_lib, dtype, cache, d, hq, hkv):
    """Lengths around the edges of groups of 16 keys, steps, blocks and pages; no rows at all; 17 rows a KV head."""
    run("token", [1, 0, 15, 16, 17, 33, 127, 128, 129, 300], hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, R=32, seed=hq)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("R", [16, 64, 128, 256])
def test_pages(gpu_lib, dtype, cache, R):
    run("pages", [R - 1, R, R + 1, 3 * R + 5, 700], hq=4, hkv=2, d=128, dtype=dtype, cache=cache, R=R, seed=R)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,new,hq,hkv,d", [(2, [2, 1, 0, 2], 2, 2, 64), (5, [5, 3, 1, 5], 8, 2, 128), (33, [33, 32, 1, 20], 3, 1, 64),
                                            (16, [16, 16, 7, 16], 8, 1, 128), (70, [70, 40, 33, 64], 1, 1, 128)])
def test_several_new_rows(gpu_lib, dtype, cache, causal, L, new, hq, hkv, d):
    """Causal and bidirectional rows, ragged counts, row blocks; prompts that are nothing but new rows."""
    run("rows", [L, 130, 64, 200], new_len=L, new=new, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, R=16, causal=causal,
        seed=L)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,new,hq,hkv,d,copies", [(1, [1, 1, 1, 1, 1], 4, 4, 64, 1), (2, [2, 1, 0, 2, 1], 2, 2, 128, 1),
                                                   (5, [5, 3, 1, 5, 0], 8, 2, 128, 1), (33, [33, 32, 1, 20, 33], 3, 1, 64, 1),
                                                   (16, [16, 16, 7, 16, 1], 8, 1, 128, 1), (2, [2, 1, 0, 2, 1], 2, 2, 64, 30)])
def test_tables_wider_than_the_sequences(gpu_lib, dtype, cache, causal, L, new, hq, hkv, d, copies):
    """Whether a call cuts its keys goes by the table's width: short sequences under a wide table and under a narrow
    one, and 300 units of them, which narrow tables of up to 2048 rows leave whole."""
    lens = [max(L, 1), 130, 64, 600, 0] * copies
    for width in (38, 400):
        run("width", lens, new_len=L, new=new * copies, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, R=16, causal=causal,
            seed=L, max_pages=width)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("lens", [[9000], [5000, 3, 0, 2500], [1000] * 9])
def test_split_keys(gpu_lib, dtype, cache, lens):
    """Long caches cut over many workgroups and joined, beside short and empty ones, and the same bits again."""
    case, c, o, lse = run("split", lens, hq=4, hkv=2, d=128, dtype=dtype, cache=cache, R=64, seed=len(lens))
    again = run_attn(case, c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_many_sequences(gpu_lib):
    """More than 64 sequences, which the plan walks in several turns; a table wider than any sequence needs."""
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 260, (150,), generator=g).tolist()
    lens[100] = 4000
    run("many", lens, hq=2, hkv=1, d=64, R=32, seed=8, max_pages=300)


@pytest.mark.parametrize("B", [129, 700, 4200])
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_batches_planned_by_a_launch_of_their_own(gpu_lib, kind, B):
    """Ragged batches with empty sequences, sequences without new rows and one long sequence, at either end of the
    batch; the same call in a graph follows other lengths."""
    dtype, cache = KINDS[kind]
    g = torch.Generator().manual_seed(B + kind)
    lens = torch.randint(0, 40, (B,), generator=g).tolist()
    lens[(0, B // 2, B - 1)[kind % 3]] = 5000
    new = [int(n) for n in torch.randint(0, 4, (B,), generator=g)]
    hq, hkv = ((4, 2), (12, 1), (3, 3))[kind % 3]                  # 12 rows, 36 (two row blocks) and 3
    case = Case(lens, new_len=3, new=new, hq=hq, hkv=hkv, d=64, dtype=dtype, cache=cache, R=16, seed=B)
    c = case.to_gpu()
    o, lse = run_attn(case, c)
    check_attn(case, o, lse)
    if B != 700:
        return
    ws = torch.empty(_lib.pd_paged_workspace_bytes(case.dims, 0, 1), dtype=torch.uint8, device="cuda")
    go, gl = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _lib.pd_paged_attn(case.dims, c["cache"], c["q"], go, gl, workspace=ws)
    for shift in (0, 100, 350):                                    # the sequences' rows in other places of the batch
        turned = {n: c[n].roll(shift, 0) for n in ("kv_len", "new_rows", "table", "q")}
        saved = {n: c[n].clone() for n in turned}
        for n, x in turned.items():
            c[n].copy_(x)
        go.fill_(7.0)
        graph.replay()
        eager, _ = run_attn(case, c)
        assert torch.equal(go, eager)
        assert shift or torch.equal(go, o)
        for n, x in saved.items():
            c[n].copy_(x)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_longer_walk_than_one_window(gpu_lib, dtype, cache):
    """Enough sequences that one workgroup walks more than 64 steps of a wave."""
    case = Case([8300], hq=2, hkv=1, d=64, dtype=dtype, cache=cache, R=16, seed=2)
    B, c = 520, case.to_gpu()                                    # all of them read the same pages
    dims = _lib.PagedDims.from_buffer_copy(case.dims)
    dims.batch = B
    wide = {n: c[n].expand(B, *c[n].shape[1:]).contiguous() for n in ("table", "q", "kv_len", "new_rows")}
    wide["kv_len"], wide["new_rows"] = (wide[n].view(-1)[:1].expand(B).contiguous() for n in ("kv_len", "new_rows"))
    cache = _lib.PagedCache(dims, c["k"], c["v"], wide["table"], wide["kv_len"], wide["new_rows"], c["k_exp"], c["v_exp"])
    o, lse = torch.empty_like(wide["q"]), torch.empty(B, 2, 1, device="cuda")
    ws = torch.empty(_lib.pd_paged_workspace_bytes(dims, 0, 1), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_attn(dims, cache, wide["q"], o, lse, workspace=ws)
    for b in (0, 77, 519):
        check_attn(case, o[b:b + 1], lse[b:b + 1])


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_large_scores(gpu_lib, dtype, cache):
    """Scores of several hundred, the largest key anywhere in the sequence: a running maximum that rises late."""
    for at in (0, 40, 900, 1499):
        case = Case([1500], hq=2, hkv=1, d=64, dtype=dtype, cache=cache, R=64, seed=at, sigma=3.0)
        case.k_rows[0][at] = (case.q[0, 0, 0] * 4).to(case.k_rows[0].dtype)
        case.place()
        c = case.to_gpu()
        check_attn(case, *run_attn(case, c))


def test_without_lse_and_unsplit_shapes(gpu_lib):
    case = Case([100, 7], hq=4, hkv=4, d=128, R=128, seed=6)     # at most one block of keys: no workspace
    assert _lib.pd_paged_workspace_bytes(case.dims, 0, 1) == 0
    c = case.to_gpu()
    o, _ = run_attn(case, c, lse=False)
    check_attn(case, o, None)


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
def test_nonfinite_values_stay_with_the_rows_that_see_them(gpu_lib, dtype, cache):
    """Values and keys that are NaN or infinite at a position that some rows see (causal): rows before it get the bits
    they get without, rows at and behind it what the formula gives."""
    for bad in ((math.nan,) if cache == PD_FP8_E4M3 else (math.nan, math.inf, -math.inf)):
        for which in ("k", "v"):
            L, hq = 6, 8
            case = Case([50], new_len=L, hq=hq, hkv=2, d=128, dtype=dtype, cache=cache, R=16, seed=12)
            clean, _ = run_attn(case, case.to_gpu())
            rows = case.k_rows if which == "k" else case.v_rows
            rows[0][47, 0, 3] = bad                               # new row 3 (of 0..5), KV head 0, channel 3
            case.place()
            o, _ = run_attn(case, case.to_gpu())
            assert torch.equal(o[:, :3], clean[:, :3]) and torch.equal(o[:, :, 4:], clean[:, :, 4:])
            hit = o[0, 3:, :4].float()
            if which == "v":
                assert torch.equal(hit[..., 4:], clean[0, 3:, :4].float()[..., 4:]) or cache == PD_FP8_E4M3
                assert torch.all(torch.isnan(hit[..., 3])) if math.isnan(bad) else torch.all(hit[..., 3] == bad)
            else:
                assert torch.all(torch.isnan(hit)) if not math.isinf(bad) else True


def test_minus_infinity_scores(gpu_lib):
    """Keys that give scores of -inf have weight zero, also where a step, a wave's keys, a part or all hold nothing
    else; then o = 0 and lse = -inf."""
    for n in (20, 700, 3000):
        case = Case([n, n], hq=1, hkv=1, d=64, R=64, seed=n)
        case.q[:, 0, 0, 0] = 1.0
        for b in range(2):
            case.k_rows[b][:, 0, 0] = -math.inf
        if n > 20:
            case.k_rows[0][n // 2, 0, 0] = 0.5
        else:
            case.k_rows[0][3, 0, 0] = 0.5
        case.place()
        c = case.to_gpu()
        o, lse = run_attn(case, c)
        torch.cuda.synchronize()
        at = n // 2 if n > 20 else 3
        assert torch.equal(o[0, 0, 0].cpu(), case.v_rows[0][at, 0])
        assert torch.all(o[1] == 0) and torch.all(lse[1] == -math.inf)


def test_bad_pages_give_nan(gpu_lib):
    """A needed page id outside the pool makes its sequence NaN and no other; a length beyond the table counts as the
    table's; entries that are not needed may hold anything."""
    for kind in KINDS:
        case = Case([100, 100, 2000], hq=4, hkv=2, d=64, dtype=kind[0], cache=kind[1], R=32, seed=3)
        c = case.to_gpu()
        good, _ = run_attn(case, c)
        c["table"][1, 2] = case.dims.n_pages
        o, lse = run_attn(case, c)
        assert torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()
        assert torch.equal(o[0], good[0]) and torch.equal(o[2], good[2])
        c["table"][1, 2] = -5
        assert torch.isnan(run_attn(case, c)[0][1]).all()


@pytest.mark.parametrize("dtype,cache", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
def test_more_new_rows_than_positions(gpu_lib, dtype, cache, causal):
    """Lengths below the number of new rows: the rows whose position lies before 0 see nothing (causal); lengths and
    counts beyond their bounds, below and above, count as the bounds."""
    case = Case([3, 64, 40], new_len=5, hq=4, hkv=2, d=64, dtype=dtype, cache=cache, R=16, causal=causal, seed=4)
    c = case.to_gpu()
    o, lse = run_attn(case, c)
    if causal:
        assert torch.all(o[0, :2] == 0) and torch.all(lse[0, :, :2] == -math.inf)
    check_attn(case, o, lse)
    c["kv_len"].copy_(torch.tensor([-9, 1 << 30, 40], dtype=torch.int32))
    c["new_rows"].copy_(torch.tensor([5, 1 << 30, -1], dtype=torch.int32))
    o, lse = run_attn(case, c)
    assert torch.all(o[0] == 0) and torch.all(lse[0] == -math.inf) and torch.all(o[2] == 7) and torch.all(lse[2] == 7)
    case.lens, case.new = [0, 64, 40], [5, 5, 0]
    case.held = {n: [case.held[n][0][:0], *case.held[n][1:]] for n in case.held}
    check_attn(case, o, lse)


def test_softmax_scale(gpu_lib):
    case = Case([77], hq=2, hkv=1, d=128, R=16, seed=5, sm_scale=0.3)
    check_attn(case, *run_attn(case, case.to_gpu()))


def test_offsets_beyond_32_bits(gpu_lib):
    """A pool of more than 2^31 elements (and bytes): pages at its end are read and written where they are."""
    R, hkv, d = 256, 8, 128
    n_pages = (1 << 31) // (R * hkv * d) + 4                     # 8196 pages, 4.3 GB each for K and V
    k = torch.zeros(n_pages, hkv, R, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    case = Case([300], hq=8, hkv=8, d=d, R=R, seed=1)
    dims = _lib.PagedDims.from_buffer_copy(case.dims)
    dims.n_pages = n_pages
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    kv, one = torch.tensor([300], dtype=torch.int32, device="cuda"), torch.tensor([300], dtype=torch.int32, device="cuda")
    dims.new_len = 300
    cache = _lib.PagedCache(dims, k, v, table, kv, one)
    _lib.pd_paged_append(dims, cache, case.k_rows[0][None].cuda(), case.v_rows[0][None].cuda())
    assert torch.equal(k[n_pages - 2, :, :44].cpu(), case.k_rows[0][256:].transpose(0, 1))
    dims.new_len = 1
    one.fill_(1)
    o, lse = torch.full_like(case.q, 7.0).cuda(), torch.empty(1, 8, 1, device="cuda")
    ws = torch.empty(_lib.pd_paged_workspace_bytes(dims, 0, 1), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_attn(dims, cache, case.q.cuda(), o, lse, workspace=ws)
    check_attn(case, o, lse)
    out = [torch.empty(1, hkv, 300, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(dims, cache, 0, 300, *out)
    assert torch.equal(out[1][0].cpu(), case.v_rows[0].transpose(0, 1))
