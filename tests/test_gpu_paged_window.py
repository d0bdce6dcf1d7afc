"""pd_paged_window_attn against float64, over a pool that holds NaN wherever no row lies, and whose pages out of sight
are in no table."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged4_case import Case4
from paged_case import HALF_STEP, Case, h64, run_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP4_E2M1, PD_FP8_E4M3

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_FP4_E2M1), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp4", "fp32"]


def make(kind, lens, **kw):
    dtype, cache = kind
    return Case4(lens, dtype=dtype, **kw) if cache == PD_FP4_E2M1 else Case(lens, dtype=dtype, cache=cache, **kw)


def run_window(case, c, window, sinks, fill=7.0, lse=True, dims=None):
    d = dims or case.dims
    o = torch.full_like(c["q"], fill)
    l = torch.full((d.batch, d.n_heads_q, d.new_len), fill, dtype=torch.float32, device=o.device) if lse else None
    nb = _lib.pd_paged_window_workspace_bytes(d, window, sinks)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device=o.device) if nb else None
    _lib.pd_paged_window_attn(d, c["cache"], c["q"], window, sinks, o, l, workspace=ws)
    return o, l


def lows(case, b, window):
    n, m, G = case.lens[b], case.new[b], case.dims.n_heads_q // case.dims.n_heads_kv
    return np.repeat([n - m + r - window + 1 for r in range(m)], G)


def hide(case, c, window, sinks):
    """Takes the pages that no row sees out of the tables: their entries lie far outside the pool."""
    R = case.dims.page_rows
    for b, n in enumerate(case.lens):
        for j in range(-(-n // R)):
            pos = np.arange(j * R, min(n, (j + 1) * R))
            if not ((pos < sinks) | (pos > n - case.new[b] - window)).any() or case.new[b] == 0:
                c["table"][b, j] = -(1 << 30)


def check(case, o, lse, window, sinks, fill=7.0):
    """Tolerances as paged_case.check_attn derives them: fp32 sums of d products, weights as bf16 terms, one rounding."""
    d = case.dims
    G, D = d.n_heads_q // d.n_heads_kv, d.head_dim
    o, lse = h64(o), None if lse is None else h64(lse)
    for b in range(d.batch):
        m = case.new[b]
        assert np.all(o[b, m:] == fill) and (lse is None or np.all(lse[b, :, m:] == fill))
        for g in range(d.n_heads_kv):
            k, v = case.held["k"][b][:, g], case.held["v"][b][:, g]
            want, l, mass, spread = ref.attn_ref(case.rows_of(b, g), k, v, case.ends(b), case.scale, None,
                                                 lows(case, b, window), sinks)
            got = o[b, :m, g * G:(g + 1) * G].reshape(-1, D)
            delta = (2 * (D + 4) * 2.0 ** -24 * spread + 2.0 ** -21 + len(k) * 2.0 ** -24)[:, None]
            tol = mass * (2 * delta + (2.0 ** -8 if d.dtype == PD_BF16 else 0)) + np.abs(want) * HALF_STEP[d.dtype] + 1e-37
            bad = ~(np.abs(got - want) <= tol)
            assert not bad.any(), (b, g, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], tol[bad][:3])
            if lse is not None:
                gl, fine = lse[b, g * G:(g + 1) * G, :m].T.reshape(-1), np.isfinite(l)
                tl = delta[:, 0] + 2.0 ** -21 * (1 + np.abs(np.where(fine, l, 0)))
                ok = (gl == l) | (fine & (np.abs(gl - np.where(fine, l, 0)) <= tl))
                assert ok.all(), (b, g, gl[~ok][:3], l[~ok][:3])


def run(name, kind, lens, window, sinks, **kw):
    print(f"[window] {name} {kind} {lens} W={window} S={sinks} {kw}", flush=True)
    case = make(kind, lens, **kw)
    c = case.to_gpu()
    hide(case, c, window, sinks)
    o, lse = run_window(case, c, window, sinks)
    torch.cuda.synchronize()
    check(case, o, lse, window, sinks)
    return case, c, o, lse


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 0), (16, 4), (17, 16), (33, 17), (128, 0), (100, 200), (299, 1),
                                          (300, 0), (1 << 30, 0), ((1 << 31) - 1, (1 << 31) - 1)])
def test_single_tokens(gpu_lib, kind, window, sinks):
    """Windows and first positions around the edges of groups of 16, wider than the sequences, overlapping."""
    run("token", kind, [1, 0, 15, 16, 17, 33, 127, 128, 129, 300], window, sinks, hq=4, hkv=2, d=64, R=16)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("hq,hkv,d,R", [(1, 1, 128, 32), (7, 1, 128, 64), (28, 4, 64, 128), (34, 2, 128, 256)])
def test_heads_and_pages(gpu_lib, kind, hq, hkv, d, R):
    run("heads", kind, [700, 20, 433], 150, 5, hq=hq, hkv=hkv, d=d, R=R, seed=hq)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (40, 0), (64, 20)])
@pytest.mark.parametrize("L,new,hq,hkv,d", [(2, [2, 1, 0, 2], 2, 2, 64), (5, [5, 3, 1, 5], 8, 2, 128), (33, [33, 32, 1, 20], 3, 1, 64),
                                            (70, [70, 40, 33, 64], 1, 1, 128), (100, [100, 9, 64, 37], 4, 2, 64)])
def test_several_new_rows(gpu_lib, kind, causal, window, sinks, L, new, hq, hkv, d):
    """Causal and bidirectional rows with windows of their own, ragged counts, row blocks, prompts of new rows alone."""
    run("rows", kind, [L, 130, 64, 200], window, sinks, new_len=L, new=new, hq=hq, hkv=hkv, d=d, R=16, causal=causal, seed=L)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("lens,window", [([9000], 8000), ([5000, 3, 0, 2500], 2100), ([1500] * 9, 1000)])
def test_split_keys(gpu_lib, kind, lens, window):
    """Windows cut over many workgroups and joined, and the same bits again."""
    case, c, o, lse = run("split", kind, lens, window, 30, hq=4, hkv=2, d=128, R=64, seed=len(lens))
    assert _lib.pd_paged_window_workspace_bytes(case.dims, window, 30) > 0
    again = run_window(case, c, window, 30)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("B", [70, 150, 700])
def test_many_sequences(gpu_lib, B):
    """More sequences than a wave walks at once, and than it walks by itself; a table wider than any needs."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 260, (B,), generator=g).tolist()
    lens[B - 20] = 4000
    for window in (90, 3000):
        run("many", KINDS[0], lens, window, 4, hq=2, hkv=1, d=64, R=32, seed=8, max_pages=300)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
def test_a_wide_window_is_no_window(gpu_lib, kind, causal):
    """The same values as pd_paged_attn up to the order of its sums, where the window holds every position."""
    case = make(kind, [900, 33, 257], new_len=3, hq=4, hkv=2, d=128, R=16, causal=causal, seed=9)
    c = case.to_gpu()
    o, lse = run_window(case, c, 900, 0)
    check(case, o, lse, 1 << 30, 0)
    p, pl = run_attn(case, c)
    assert torch.allclose(lse, pl, rtol=2.0 ** -20, atol=2.0 ** -20)
    tol = 4 * HALF_STEP[case.dims.dtype] if case.dims.dtype == PD_BF16 else 2.0 ** -18
    assert torch.allclose(o.float(), p.float(), rtol=tol, atol=tol)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("which", ["k", "v"])
def test_nonfinite_rows_stay_with_the_rows_that_see_them(gpu_lib, kind, causal, which):
    """A NaN or an infinity at a position: rows whose window does not hold it keep their bits, before it (causal) and
    behind it; the others are NaN, or infinite, as the formula has it."""
    L, W, n = 12, 5, 60                                # row r is position 48 + r and sees (43 + r, ...]
    for bad in ((math.nan,) if kind[1] in (PD_FP8_E4M3, PD_FP4_E2M1) else (math.nan, math.inf, -math.inf)):
        for at in (46, 52):
            case = make(kind, [n], new_len=L, hq=8, hkv=2, d=64, R=16, causal=causal, seed=12)
            clean, _ = run_window(case, case.to_gpu(), W, 2)
            rows = case.k_rows if which == "k" else case.v_rows
            rows[0][at, 0, 3] = bad
            case.place()
            o, _ = run_window(case, case.to_gpu(), W, 2)
            own = np.arange(n - L, n)
            sees = ((at <= own) if causal else (at < n)) & (at > own - W)
            far = torch.from_numpy(np.flatnonzero(~sees))
            assert torch.equal(o[:, far], clean[:, far]) and torch.equal(o[:, :, 4:], clean[:, :, 4:])
            hit = o[0, torch.from_numpy(np.flatnonzero(sees)), :4].float()
            if which == "v":
                x = hit[..., 3]
                assert torch.isnan(x).all() if math.isnan(bad) else torch.all(x == bad)
            elif math.isnan(bad):
                assert torch.isnan(hit).all()


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_bad_pages_and_hidden_ones(gpu_lib, kind):
    """A page id outside the pool makes the rows NaN that see one of its positions, and no others: rows before it, rows
    whose window lies behind it, other sequences."""
    L, W = 40, 10
    case = make(kind, [100, 100, 300], new_len=L, hq=4, hkv=2, d=64, R=16, seed=3)
    c = case.to_gpu()
    good, gl = run_window(case, c, W, 3)
    for page in (case.dims.n_pages, -5):
        c["table"][1, 5] = page                       # positions 80..95; rows 20.. of 60.. see it, until row 44
        o, lse = run_window(case, c, W, 3)
        assert torch.equal(o[0], good[0]) and torch.equal(o[2], good[2])
        assert torch.equal(o[1, :20], good[1, :20]) and torch.isnan(o[1, 20:]).all()
        assert torch.isnan(lse[1, :, 20:]).all() and torch.equal(lse[1, :, :20], gl[1, :, :20])
        c["table"][1, 5] = case.table[1, 5].item()
        c["table"][1, 4] = page                       # 64..79; rows 4..28 see it
        o, _ = run_window(case, c, W, 3)
        assert torch.isnan(o[1, 4:29]).all() and torch.equal(o[1, :4], good[1, :4]) and torch.equal(o[1, 29:], good[1, 29:])
        c["table"][1, 4] = case.table[1, 4].item()
        c["table"][1, 0] = page                       # the first positions: every row
        assert torch.isnan(run_window(case, c, W, 3)[0][1]).all()
        assert torch.equal(run_window(case, c, W, 0)[0][0], run_window(case, c, W, 0)[0][0])
        c["table"][1, 0] = case.table[1, 0].item()


def test_minus_infinity_scores(gpu_lib):
    """Keys that give scores of -inf have weight zero, also where the window holds nothing else."""
    case = Case([200, 200], hq=1, hkv=1, d=64, R=64, seed=1)
    case.q[:, 0, 0, 0] = 1.0
    for b in range(2):
        case.k_rows[b][:, 0, 0] = -math.inf
    case.k_rows[0][150, 0, 0] = 0.5
    case.place()
    o, lse = run_window(case, case.to_gpu(), 60, 3)
    assert torch.equal(o[0, 0, 0].cpu(), case.v_rows[0][150, 0]) and torch.all(o[1] == 0) and torch.all(lse[1] == -math.inf)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("causal", [0, 1])
def test_more_new_rows_than_positions(gpu_lib, kind, causal):
    case = make(kind, [3, 64, 40], new_len=5, hq=4, hkv=2, d=64, R=16, causal=causal, seed=4)
    c = case.to_gpu()
    o, lse = run_window(case, c, 2, 1)
    check(case, o, lse, 2, 1)
    if causal:
        assert torch.all(o[0, :2] == 0) and torch.all(lse[0, :, :2] == -math.inf)
    c["kv_len"].copy_(torch.tensor([-9, 1 << 30, 40], dtype=torch.int32))
    c["new_rows"].copy_(torch.tensor([5, 1 << 30, -1], dtype=torch.int32))
    o, lse = run_window(case, c, 2, 1)
    assert torch.all(o[0] == 0) and torch.all(lse[0] == -math.inf) and torch.all(o[2] == 7) and torch.all(lse[2] == 7)
    case.lens, case.new = [0, 64, 40], [5, 5, 0]
    case.held = {n: [case.held[n][0][:0], *case.held[n][1:]] for n in case.held}
    check(case, o, lse, 2, 1)


def test_without_lse_and_without_workspace(gpu_lib):
    """A window of a few blocks is never cut, however long the table: no workspace."""
    case = Case([1000, 7], hq=4, hkv=4, d=128, R=128, seed=6, max_pages=1000)
    assert _lib.pd_paged_window_workspace_bytes(case.dims, 64, 4) == 0
    o, _ = run_window(case, case.to_gpu(), 64, 4, lse=False)
    check(case, o, None, 64, 4)


@pytest.mark.parametrize("kind", KINDS[:2], ids=IDS[:2])
def test_graph_follows_the_lengths(gpu_lib, kind):
    """Captured once, replayed among eager calls while the sequences grow: the bits of the eager call every time."""
    case = make(kind, [700, 1200, 90], hq=4, hkv=2, d=128, R=16, seed=5)
    c = case.to_gpu()
    ws = torch.empty(_lib.pd_paged_window_workspace_bytes(case.dims, 600, 4) + 16, dtype=torch.uint8, device="cuda")
    o, l = torch.zeros_like(c["q"]), torch.zeros(3, 4, 1, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            _lib.pd_paged_window_attn(case.dims, c["cache"], c["q"], 600, 4, o, l, workspace=ws)
    torch.cuda.synchronize()
    for cut in (0, 1, 40, 89, 0):
        c["kv_len"].copy_(torch.tensor([n - cut for n in case.lens], dtype=torch.int32))
        eager = run_window(case, c, 600, 4)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager[0]) and torch.equal(l, eager[1])


def test_long_caches(gpu_lib):
    """Positions of 2^20 and more under a small window: as much is read as for a short cache, at the offsets of the end."""
    n, R, W = (1 << 20) + 77, 256, 300
    case = Case([n - (n - 333) // R * R], hq=4, hkv=2, d=64, R=R, seed=2)      # the rows of the last pages
    first = (n - case.lens[0]) // R
    c = case.to_gpu()
    table = torch.full((1, first + 3), -9, dtype=torch.int32, device="cuda")
    pages = -(-case.lens[0] // R)
    table[0, first:first + pages] = c["table"][0, :pages]
    dims = _lib.PagedDims.from_buffer_copy(case.dims)
    dims.max_pages = table.shape[1]
    kv = torch.tensor([n], dtype=torch.int32, device="cuda")
    c["cache"] = _lib.PagedCache(dims, c["k"], c["v"], table, kv, c["new_rows"])
    o, lse = run_window(case, c, W, 0, dims=dims)
    check(case, o, lse, W, 0)


@pytest.mark.parametrize("L", [1, 40])
def test_two_calls_at_once(gpu_lib, L):
    """Two streams, each with a cache, outputs and a workspace of its own, over and over: the bits of a call alone."""
    cases = [make(KINDS[i], [900 + 300 * i, 1500, 77], new_len=L, hq=16, hkv=4, d=128, R=16, seed=20 + i) for i in range(2)]
    held = [case.to_gpu() for case in cases]
    want = [run_window(case, c, 700, 4) for case, c in zip(cases, held)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(_lib.pd_paged_window_workspace_bytes(case.dims, 700, 4) + 16, dtype=torch.uint8, device="cuda") for case in cases]
    outs = [[(torch.full_like(w[0], 7.0), torch.full_like(w[1], 7.0)) for _ in range(20)] for w in want]
    torch.cuda.synchronize()
    for i in range(20):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                o, l = outs[s][i]
                _lib.pd_paged_window_attn(cases[s].dims, held[s]["cache"], held[s]["q"], 700, 4, o, l, workspace=ws[s])
    torch.cuda.synchronize()
    for s in range(2):
        assert all(torch.equal(o, want[s][0]) and torch.equal(l, want[s][1]) for o, l in outs[s])
