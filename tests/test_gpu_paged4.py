"""A paged cache in 4 bits: rows written (every bit of the pool against the oracle), read back, and attended to, over a
pool that holds NaN wherever no row lies."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged4_case import Case4, unpack4
from paged_case import check_attn, h64, run_attn
from paper_2606_10537_amd import _lib
from test_gpu_paged_cache import append_all

pytestmark = pytest.mark.gpu


def empty_pool(case):
    for n in ("k", "v"):
        case.pool[n], case.pool[n + "_exp"] = torch.full_like(case.pool[n], 0x77), torch.full_like(case.pool[n + "_exp"], 255)
    case.pool["bounds"] = torch.full_like(case.pool["bounds"], math.nan)
    return case.to_gpu()


@pytest.mark.parametrize("R,L,lens,d,hkv", [(16, 1, [1, 3, 17, 0], 64, 2), (16, 33, [33, 5, 64, 0, 47], 128, 1),
                                            (64, 70, [131, 64, 1], 128, 3), (256, 300, [300, 256, 511], 64, 2),
                                            (32, 7, [40, 32, 31], 128, 4)])
def test_append_writes_every_row_and_nothing_else(gpu_lib, R, L, lens, d, hkv):
    print(f"[append4] R={R} L={L} lens={lens}", flush=True)
    case = Case4(lens, new_len=L, hq=hkv, hkv=hkv, d=d, R=R, seed=R + L)
    want = {k: v.clone() for k, v in case.pool.items()}
    c = empty_pool(case)
    append_all(case, c, max(-(-n // L) for n in lens), stride_extra=1)
    for n in ("k", "v", "k_exp", "v_exp"):
        assert torch.equal(c[n].cpu(), want[n]), n
    assert torch.equal(c["bounds"].cpu().view(torch.int16), want["bounds"].view(torch.int16))


@pytest.mark.parametrize("d", [64, 128])
def test_append_and_read_of_special_values(gpu_lib, d):
    """Rows of zeros, of one value at every power of two, of every border between neighbours, subnormal, huge, with NaN
    and infinities: the oracle's bytes, and read back what they stand for."""
    n = 130
    case = Case4([n], new_len=n, hq=1, hkv=1, d=d, R=64, seed=3)
    x = case.k_rows[0]
    for i in range(60):
        x[i] *= 2.0 ** (4 * i - 120)
    x[60] = 0
    x[61] = -0.0
    borders = torch.tensor([(a + b) / 2 for a, b in zip(ref.E2M1, ref.E2M1[1:])])
    for i in range(8):                                # codes, borders, and the bf16 neighbours of both sides
        row = torch.cat([torch.tensor(ref.E2M1), borders, borders * (1 + 2.0 ** -7), borders * (1 - 2.0 ** -8)]).float()[:29]
        x[62 + i, 0, :29] = (row * 2.0 ** (i - 4) * (1 if i % 2 else -1)).to(x.dtype)
        x[62 + i, 0, 29:] = 6.0 * 2.0 ** (i - 4)
    x[70, 0, 3] = math.inf
    x[71, 0, 34] = -math.inf
    x[72, 0, 5] = math.nan
    x[73] = math.nan
    x[74] = 3.3e38
    x[75] = torch.finfo(torch.bfloat16).max
    x[76] = 1e-40
    x[77, 0, :32] = 2.0 ** -101                        # below the least power of two's half step: zeros, or 0.5 * 2^-100
    x[77, 0, 1] = 2.0 ** -102
    x[78, 0, :32] = 1.5 * 2.0 ** 127
    x[79, 0, :32] = 1.75 * 2.0 ** 127
    c = empty_pool(case)
    k = x[None].cuda()
    _lib.pd_paged_append(case.dims, c["cache"], k, k)
    codes, e = ref.quantise4_ref(h64(x))
    pages = [int(case.table[0, j]) for j in range(3)]
    ge = torch.cat([c["k_exp"][p] for p in pages], 2)[0, :, :n].cpu().numpy().astype(int) - 127
    assert np.array_equal(ge.T, e[:, 0])
    fine = np.repeat(e[:, 0] != 128, 32, -1)
    got = unpack4(torch.cat([c["k"][p] for p in pages], 1)[0, :n].cpu().numpy())
    assert np.array_equal(got[fine], codes[:, 0][fine])
    out = [torch.full((1, 1, n, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(case.dims, c["cache"], 0, n, *out)
    held = ref.held4_ref(codes, e)[:, 0]
    with np.errstate(invalid="ignore"):
        held = np.where(np.abs(held) >= 2.0 ** 128, np.sign(held) * np.inf, held)
    for o in out:
        np.testing.assert_array_equal(h64(o)[0, 0], held)


@pytest.mark.parametrize("R,d,first,count", [(16, 64, 0, 77), (64, 128, 30, 100), (256, 128, 255, 3), (16, 128, 0, 1)])
def test_read(gpu_lib, R, d, first, count):
    """Ragged sequences, rows behind them left as they were, a page id outside the pool."""
    case = Case4([77, 3, 0, 300], hq=2, hkv=2, d=d, R=R, seed=R, max_pages=20)
    c = case.to_gpu()
    out = [torch.full((4, 2, count, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(case.dims, c["cache"], first, count, *out)
    for n, o in zip("kv", out):
        want = np.full((4, 2, count, d), 7.0)
        for b in range(4):
            rows = case.held[n][b][first:first + count]
            want[b, :, :len(rows)] = rows.transpose(1, 0, 2)
        np.testing.assert_array_equal(h64(o), want)
    c["table"][3, first // R] = case.dims.n_pages
    _lib.pd_paged_read(case.dims, c["cache"], first, count, *out)
    assert torch.isnan(out[0][3, :, 0]).all() and torch.equal(out[0][:3].cpu(), torch.from_numpy(np.array(h64(out[0][:3]))).to(torch.bfloat16))


def run(name, *a, **kw):
    print(f"[attn4] {name} {a} {kw}", flush=True)
    case = Case4(*a, **kw)
    c = case.to_gpu()
    o, lse = run_attn(case, c)
    torch.cuda.synchronize()
    check_attn(case, o, lse)
    return case, c, o, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (7, 1), (16, 2), (28, 4), (34, 2)])
def test_single_tokens(gpu_lib, d, hq, hkv):
    """Lengths around the edges of groups of 16 keys, steps, blocks and pages; no rows at all; 17 rows a KV head."""
    run("token", [1, 0, 15, 16, 17, 33, 127, 128, 129, 300], hq=hq, hkv=hkv, d=d, R=32, seed=hq)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("R", [16, 64, 128, 256])
def test_pages(gpu_lib, R, d):
    run("pages", [R - 1, R, R + 1, 3 * R + 5, 700], hq=4, hkv=2, d=d, R=R, seed=R)


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("L,new,hq,hkv,d", [(2, [2, 1, 0, 2], 2, 2, 64), (5, [5, 3, 1, 5], 8, 2, 128), (33, [33, 32, 1, 20], 3, 1, 64),
                                            (16, [16, 16, 7, 16], 8, 1, 128), (70, [70, 40, 33, 64], 1, 1, 128)])
def test_several_new_rows(gpu_lib, causal, L, new, hq, hkv, d):
    run("rows", [L, 130, 64, 200], new_len=L, new=new, hq=hq, hkv=hkv, d=d, R=16, causal=causal, seed=L)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[9000], [5000, 3, 0, 2500], [1000] * 9])
def test_split_keys(gpu_lib, lens, d):
    """Long caches cut over many workgroups and joined, and the same bits again."""
    case, c, o, lse = run("split", lens, hq=4, hkv=2, d=d, R=64, seed=len(lens))
    again = run_attn(case, c)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_many_sequences(gpu_lib):
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 260, (150,), generator=g).tolist()
    lens[100] = 4000
    run("many", lens, hq=2, hkv=1, d=64, R=32, seed=8, max_pages=300)


@pytest.mark.parametrize("causal", [0, 1])
def test_chosen_pages(gpu_lib, causal):
    """Pages chosen by bounds on the scores of the keys as they were given; entries outside the table are skipped."""
    case = Case4([300, 40, 0, 1000], new_len=2, hq=4, hkv=2, d=128, R=16, seed=2, causal=causal, max_pages=64)
    case.new = [2, 2, 0, 1]
    c = case.to_gpu()
    idx = torch.zeros(4, 2, 5, dtype=torch.int32, device="cuda")
    ws = torch.empty(_lib.pd_paged_workspace_bytes(case.dims, 5, 0), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_select(case.dims, c["cache"], c["q"], 5, 1, 1, idx, ws)
    assert idx[0].min() >= 0 and idx[2].max() == -1
    idx[3, 0, 2] = -7
    check_attn(case, *run_attn(case, c, page_idx=idx), page_idx=idx.cpu())


@pytest.mark.parametrize("which", ["k", "v"])
def test_groups_that_are_nan_stay_with_the_rows_that_see_them(gpu_lib, which):
    """A NaN makes its 32 channels of the row NaN: causal rows before it keep their bits; behind it a key makes the whole
    row NaN, a value those channels."""
    case = Case4([50], new_len=6, hq=8, hkv=2, d=128, R=16, seed=12)
    clean, _ = run_attn(case, case.to_gpu())
    (case.k_rows if which == "k" else case.v_rows)[0][47, 0, 37] = math.nan
    case.place()
    o, _ = run_attn(case, case.to_gpu())
    assert torch.equal(o[:, :3], clean[:, :3]) and torch.equal(o[:, :, 4:], clean[:, :, 4:])
    hit = o[0, 3:, :4].float()
    assert torch.isnan(hit[..., 32:64]).all()
    rest = torch.cat([hit[..., :32], hit[..., 64:]], -1)
    assert torch.isnan(rest).all() if which == "k" else torch.equal(rest, torch.cat([clean[0, 3:, :4, :32], clean[0, 3:, :4, 64:]], -1).float())


def test_bad_pages_give_nan(gpu_lib):
    case = Case4([100, 100, 2000], hq=4, hkv=2, d=64, R=32, seed=3)
    c = case.to_gpu()
    good, _ = run_attn(case, c)
    for page in (case.dims.n_pages, -5):
        c["table"][1, 2] = page
        o, lse = run_attn(case, c)
        assert torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()
        assert torch.equal(o[0], good[0]) and torch.equal(o[2], good[2])


def test_large_scores(gpu_lib):
    """Scores of several hundred, the largest key anywhere in the sequence: a running maximum that rises late."""
    for at in (0, 40, 900, 1499):
        case = Case4([1500], hq=2, hkv=1, d=64, R=64, seed=at, sigma=3.0)
        case.k_rows[0][at] = (case.q[0, 0, 0] * 4).to(case.k_rows[0].dtype)
        case.place()
        check_attn(case, *run_attn(case, case.to_gpu()))


def test_offsets_beyond_32_bits(gpu_lib):
    """A pool of more than 2^32 bytes: pages at its end are written, read and attended to where they are."""
    R, hkv, d = 256, 8, 128
    n_pages = (1 << 32) // (R * hkv * d // 2) + 4                   # 32772 pages
    case = Case4([300], hq=8, hkv=8, d=d, R=R, seed=1)
    k, v = (torch.zeros(n_pages, hkv, R, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
    ke, ve = (torch.zeros(n_pages, hkv, d // 32, R, dtype=torch.uint8, device="cuda") for _ in range(2))
    dims = _lib.PagedDims.from_buffer_copy(case.dims)
    dims.n_pages, dims.new_len = n_pages, 300
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    kv, new = (torch.tensor([300], dtype=torch.int32, device="cuda") for _ in range(2))
    cache = _lib.PagedCache(dims, k, v, table, kv, new, ke, ve)
    _lib.pd_paged_append(dims, cache, case.k_rows[0][None].cuda(), case.v_rows[0][None].cuda())
    out = [torch.empty(1, hkv, 300, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(dims, cache, 0, 300, *out)
    for n, o in zip("kv", out):
        np.testing.assert_array_equal(h64(o)[0], case.held[n][0].transpose(1, 0, 2))
    dims.new_len = 1
    new.fill_(1)
    o, lse = torch.full_like(case.q, 7.0).cuda(), torch.empty(1, 8, 1, device="cuda")
    ws = torch.empty(_lib.pd_paged_workspace_bytes(dims, 0, 1), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_attn(dims, cache, case.q.cuda(), o, lse, workspace=ws)
    check_attn(case, o, lse)
