"""pd_paged_append_rope: query rows and every bit of the pool, written or not, against the oracle's norms and rotations
rounded to fp32 and to the element type; and a run of it with the calls that read the pages."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged4_case import Case4
from paged_case import TORCH, Case, check_attn, h64, run_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP4_E2M1, PD_FP8_E4M3
from test_gpu_paged_window import check as check_window, run_window

pytestmark = pytest.mark.gpu
KINDS = [(PD_BF16, PD_BF16), (PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_FP4_E2M1), (PD_FP32, PD_FP32)]
IDS = ["bf16", "fp8", "fp4", "fp32"]
BASE, EPS = 5e5, 1e-6
# Both sides evaluate in double and round to fp32: an fp32 result is off by one rounding, where the value lies next to the
# border of two numbers.  An angle a = pos * f has three roundings of 2^-53 of itself on either side (f, the product, the
# reduction), 2^-50 |a| in all, |a| <= 200000 here, and an element moves by that times its partner, below 8: where the two terms
# of a rotation cancel, this is more than a rounding of the result.  A bf16 one changes only where the value in double
# lies within as much of a border, about once in 2^20 elements of 2^-10 and less.
ONE_ANGLE = 200000 * 2.0 ** -50 * 8
ONE_FP32 = 2.0 ** -23


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x)).float().to(TORCH[dtype])


class Rows:
    """Projected rows for every position of a case's sequences, and what they become: sets the case's rows."""

    def __init__(self, kind, lens, norm=True, rotate=True, given=False, seed=0, sigma=1.5, **kw):
        dtype, cache = kind
        self.case = case = (Case4 if cache == PD_FP4_E2M1 else Case)(lens, dtype=dtype, seed=seed, **dict(kw, **({} if cache == PD_FP4_E2M1 else {"cache": cache})))
        d, g, t = case.dims, case.g, TORCH[dtype]
        self.base = BASE if rotate else 0.0
        heads = d.n_heads_q + 2 * d.n_heads_kv
        self.x = [(torch.randn(n, heads, d.head_dim, generator=g) * sigma).to(t) for n in lens]
        self.w = [(1 + 0.2 * torch.randn(d.head_dim, generator=g)).to(t) if norm else None for _ in range(2)]
        self.pos = [torch.randint(-200000, 200000, (n,), generator=g, dtype=torch.int32) if given else torch.arange(n, dtype=torch.int32) for n in lens]
        self.given = given
        self.turn()

    def turn(self):
        case, d = self.case, self.case.dims
        hq, hkv = d.n_heads_q, d.n_heads_kv
        w = [None if x is None else h64(x) for x in self.w]
        with np.errstate(invalid="ignore", divide="ignore"):
            self.q = [ref.qk_norm_rope_ref(h64(x)[:, :hq], w[0], EPS, p.numpy(), self.base) for x, p in zip(self.x, self.pos)]
            k = [ref.qk_norm_rope_ref(h64(x)[:, hq:hq + hkv], w[1], EPS, p.numpy(), self.base) for x, p in zip(self.x, self.pos)]
        case.k_rows = [rounded(x, d.dtype) for x in k]
        case.v_rows = [x[:, hq + hkv:].contiguous() for x in self.x]
        case.place()

    def empty(self):
        case = self.case
        for n in ("k", "v", "k_exp", "v_exp", "bounds"):
            if case.pool[n] is not None:
                t = case.pool[n]
                case.pool[n] = torch.full_like(t, (0x7F if case.fp8 else 0x77) if n in "kv" and t.dtype is torch.uint8 else 255 if t.dtype is torch.uint8 else math.nan)
        return case.to_gpu()

    def call(self, c, first, new, extra=0, with_q=True, q_out=None, dims=None, stream=None):
        """Rows first[b] .. first[b] + new[b] of every sequence; NaN in the places of no row."""
        d = dims or self.case.dims
        L, hq, hkv = d.new_len, d.n_heads_q, d.n_heads_kv
        fused = torch.full((d.batch, L, hq + 2 * hkv + extra, d.head_dim), math.nan, dtype=TORCH[d.dtype])
        pos = torch.full((d.batch, L), 1 << 30, dtype=torch.int32)
        for b, (f, m) in enumerate(zip(first, new)):
            fused[b, :m, :hq + 2 * hkv] = self.x[b][f:f + m]
            pos[b, :m] = self.pos[b][f:f + m]
        fused = fused.cuda()
        c["kv_len"].copy_(torch.tensor([f + m for f, m in zip(first, new)], dtype=torch.int32))
        c["new_rows"].copy_(torch.tensor(new, dtype=torch.int32))
        q = fused[:, :, :hq] if with_q else None
        if with_q and q_out is None:
            q_out = torch.full((d.batch, L, hq, d.head_dim), 7.0, dtype=TORCH[d.dtype], device="cuda")
        _lib.pd_paged_append_rope(d, c["cache"], q, fused[:, :, hq:hq + hkv], fused[:, :, hq + hkv:hq + 2 * hkv], self.w[0] if self.w[0] is None else self.w[0].cuda(),
                                  self.w[1] if self.w[1] is None else self.w[1].cuda(), EPS, pos.cuda() if self.given else None, self.base, q_out if with_q else None, stream=stream)
        return q_out

    def check_q(self, out, first, new, fill=7.0):
        d = self.case.dims
        out = out.cpu()
        for b, (f, m) in enumerate(zip(first, new)):
            assert torch.all(out[b, m:] == fill)
            same(out[b, :m], rounded(self.q[b][f:f + m], d.dtype))


def same(got, want):
    if got.dtype is torch.float32:
        got, want = got.double(), want.double()
        off = (got - want).abs()
        assert torch.all((off <= ONE_FP32 * want.abs() + ONE_ANGLE) | (torch.isnan(got) & torch.isnan(want)) | (got == want))
        return
    if got.dtype is torch.bfloat16:
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        got, want = got.nan_to_num(), want.nan_to_num()
    bad = got != want
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


def check_pool(case, c, want):
    for n in ("k", "v", "k_exp", "v_exp", "bounds"):
        if want[n] is not None:
            print(f"[pool] {n}", flush=True)
            same(c[n].cpu(), want[n])


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("R,L,lens,d,hq,hkv", [(16, 1, [1, 3, 17, 0], 64, 2, 2), (16, 33, [33, 5, 64, 0, 47], 128, 4, 1),
                                               (64, 70, [131, 64, 1], 128, 3, 3), (256, 300, [300, 256, 511], 64, 2, 2),
                                               (32, 7, [40, 32, 31], 128, 28, 4), (128, 130, [129, 1], 128, 17, 17)])
def test_every_row_and_nothing_else(gpu_lib, kind, R, L, lens, d, hq, hkv):
    print(f"[rope] {kind} R={R} L={L} lens={lens} {hq}/{hkv} d={d}", flush=True)
    for given in (False, True):
        rows = Rows(kind, lens, given=given, new_len=L, hq=hq, hkv=hkv, d=d, R=R, seed=R + L)
        case = rows.case
        want = dict(case.pool)
        c = rows.empty()
        done = [0] * len(lens)
        while done != lens:
            new = [min(L, n - at) for n, at in zip(lens, done)]
            rows.check_q(rows.call(c, done, new, extra=1), done, new)
            done = [a + b for a, b in zip(done, new)]
        check_pool(case, c, want)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("norm,rotate,with_q", [(True, False, True), (False, True, True), (False, False, True), (True, True, False)])
def test_parts_of_it(gpu_lib, kind, norm, rotate, with_q):
    """No norm, no rotation, no query rows."""
    lens = [37, 64, 1]
    rows = Rows(kind, lens, norm=norm, rotate=rotate, new_len=64, hq=6, hkv=2, d=128, R=16, seed=2)
    want = dict(rows.case.pool)
    c = rows.empty()
    out = rows.call(c, [0] * 3, lens, with_q=with_q)
    if with_q:
        rows.check_q(out, [0] * 3, lens)
    check_pool(rows.case, c, want)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("d", [64, 128])
def test_the_bits_of_append(gpu_lib, kind, d):
    """Without norm and rotation: what pd_paged_append writes, for rows with zeros, subnormals, NaN and infinities."""
    n = 50
    rows = Rows(kind, [n], norm=False, rotate=False, new_len=n, hq=2, hkv=2, d=d, R=16, seed=6)
    x = rows.x[0]
    for i in range(20):
        x[i] *= 2.0 ** (12 * i - 120)
    x[20], x[21], x[22] = 0, -0.0, 1e-40
    x[23, :, 5], x[24, :, 40], x[25, :, 6], x[26] = math.inf, -math.inf, math.nan, math.nan
    x[27] = 3.3e38
    c = rows.empty()
    out = rows.call(c, [0], [n])
    e = rows.empty()
    e["kv_len"].copy_(c["kv_len"])
    e["new_rows"].copy_(c["new_rows"])
    g = x[None].cuda()
    _lib.pd_paged_append(rows.case.dims, e["cache"], g[:, :, 2:4], g[:, :, 4:])
    bits = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])  # noqa: E731
    assert torch.equal(bits(out), bits(g[:, :, :2].contiguous()))
    for name in ("k", "v", "k_exp", "v_exp", "bounds"):
        if c[name] is not None:
            assert torch.equal(bits(c[name]), bits(e[name])), name


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_special_rows_under_norm_and_rotation(gpu_lib, kind):
    """Zeros (0 with eps), tiny and huge rows (their squares pass fp32), NaN and infinities: as the formula in double."""
    n = 12
    rows = Rows(kind, [n], new_len=n, hq=3, hkv=3, d=128, R=16, seed=7)
    x = rows.x[0]
    x[0], x[2, :6], x[3, :6] = 0, 3e38, -1e-30
    x[4, :6, 10], x[5, :6, 100], x[6, :6, 70] = math.nan, math.inf, -math.inf
    x[7, :6] *= 1e30
    rows.turn()
    held = rows.case.held
    c = rows.empty()
    out = rows.call(c, [0], [n])
    rows.check_q(out, [0], [n])
    got = [torch.zeros(1, 3, n, 128, dtype=TORCH[kind[0]], device="cuda") for _ in range(2)]
    _lib.pd_paged_read(rows.case.dims, c["cache"], 0, n, *got)      # NaN has more than one code in the pages
    tol = dict(rtol=ONE_FP32, atol=ONE_ANGLE) if kind[0] == PD_FP32 else dict(rtol=0, atol=0)
    for name, x in zip("kv", got):
        np.testing.assert_allclose(h64(x)[0], held[name][0].transpose(1, 0, 2), **tol)


@pytest.mark.parametrize("kind", KINDS[::3], ids=IDS[::3])
def test_queries_in_place_and_far_positions(gpu_lib, kind):
    """q_out is q; positions over the whole range of int32, whose angles are reduced in double."""
    lens, L, hq, d = [5, 9], 9, 4, 64
    rows = Rows(kind, lens, given=True, new_len=L, hq=hq, hkv=2, d=d, R=16, seed=8)
    rows.pos = [torch.tensor([(1 << 31) - 1, -(1 << 31), 131071, 7, -1], dtype=torch.int32), torch.randint(-(1 << 31), (1 << 31) - 1, (9,), generator=rows.case.g, dtype=torch.int64).int()]
    rows.turn()
    c = rows.empty()
    t = TORCH[kind[0]]
    q = torch.full((2, L, hq, d), 7.0, dtype=t)
    kv = torch.zeros(2, L, 4, d, dtype=t)
    pos = torch.zeros(2, L, dtype=torch.int32)
    for b in range(2):
        q[b, :lens[b]], kv[b, :lens[b]], pos[b, :lens[b]] = rows.x[b][:, :hq], rows.x[b][:, hq:], rows.pos[b]
    q, kv = q.cuda(), kv.cuda()
    c["kv_len"].copy_(torch.tensor(lens, dtype=torch.int32))
    c["new_rows"].copy_(torch.tensor(lens, dtype=torch.int32))
    _lib.pd_paged_append_rope(rows.case.dims, c["cache"], q, kv[:, :, :2], kv[:, :, 2:], rows.w[0].cuda(), rows.w[1].cuda(), EPS, pos.cuda(), BASE, q)
    # An angle of up to 2^31 is off by its own roundings in double on both sides: 2^31 * 2^-51 of a turn and less, which is
    # 2^-18 of an element's size (the head's elements are below 8).
    got = h64(q)
    for b in range(2):
        off = np.abs(got[b, :lens[b]] - rows.q[b])
        assert np.all(off <= 8 * 2.0 ** -18 + np.abs(rows.q[b]) * (2.0 ** -8 if kind[0] == PD_BF16 else 2.0 ** -24))
        assert np.all(got[b, lens[b]:] == 7.0)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_positions_below_zero_and_bad_pages(gpu_lib, kind):
    """Fewer positions than new rows: the first rows go nowhere but their queries; a page id outside the pool is not
    written to, and the queries of its rows are."""
    L = 40
    rows = Rows(kind, [60, 60, 60], given=True, new_len=L, hq=4, hkv=2, d=128, R=16, seed=9)
    case, want = rows.case, None
    c = rows.empty()
    before = {n: c[n].clone() for n in ("k", "v", "k_exp", "v_exp", "bounds") if c[n] is not None}
    d = case.dims
    fused = torch.stack([rows.x[b][:L] for b in range(3)]).cuda()
    pos = torch.stack([rows.pos[b][:L] for b in range(3)]).cuda()
    c["kv_len"].copy_(torch.tensor([10, 0, 40], dtype=torch.int32))     # rows 30.. are positions 0..; none; all
    c["new_rows"].copy_(torch.tensor([L, L, L], dtype=torch.int32))
    c["table"][2, 1] = d.n_pages + 3                                    # positions 16..31
    c["table"][1, 0] = -1
    out = torch.full((3, L, 4, 128), 7.0, dtype=TORCH[d.dtype], device="cuda")
    _lib.pd_paged_append_rope(d, c["cache"], fused[:, :, :4], fused[:, :, 4:6], fused[:, :, 6:], rows.w[0].cuda(), rows.w[1].cuda(), EPS, pos, BASE, out)
    torch.cuda.synchronize()
    for b in range(3):
        same(out[b].cpu(), rounded(rows.q[b][:L], d.dtype))
    got = [torch.zeros(3, 2, 48, 128, dtype=TORCH[d.dtype], device="cuda") for _ in range(2)]
    _lib.pd_paged_read(d, c["cache"], 0, 48, *got)
    k = h64(got[0])
    assert np.isnan(k[2, :, 16:32]).all()
    tol = dict(rtol=ONE_FP32, atol=ONE_ANGLE) if kind[0] == PD_FP32 else dict(rtol=0, atol=0)
    np.testing.assert_allclose(k[0, :, :10], case.held["k"][0][30:40].transpose(1, 0, 2), **tol)
    np.testing.assert_allclose(k[2, :, :16], case.held["k"][2][:16].transpose(1, 0, 2), **tol)
    np.testing.assert_allclose(k[2, :, 32:40], case.held["k"][2][32:40].transpose(1, 0, 2), **tol)
    touched = {int(case.table[0, 0]), int(case.table[2, 0]), int(case.table[2, 2])}
    rest = [p for p in range(d.n_pages) if p not in touched]
    for n, old in before.items():
        assert torch.equal(c[n][rest].view(torch.uint8), old[rest].view(torch.uint8)), n


@pytest.mark.parametrize("kind", KINDS[:1] + KINDS[3:], ids=IDS[:1] + IDS[3:])
def test_bounds_are_widened(gpu_lib, kind):
    """A page begins anew with its row 0 and is widened otherwise; NaNs do not count; no bounds: none are written."""
    rows = Rows(kind, [40], new_len=40, hq=2, hkv=2, d=64, R=32, seed=10)
    rows.x[0][3, 2:4, 7] = math.nan
    rows.turn()
    d1 = _lib.PagedDims.from_buffer_copy(rows.case.dims)
    c = rows.empty()
    k = torch.where(torch.isnan(rows.case.k_rows[0]), torch.tensor(0.0, dtype=rows.case.k_rows[0].dtype), rows.case.k_rows[0]).float()
    nan = torch.isnan(rows.case.k_rows[0])
    low, high = (torch.where(nan, torch.tensor(s * math.inf), k) for s in (1, -1))
    for first, m in ((0, 20), (20, 1), (21, 19)):
        rows.call(c, [first], [m], dims=d1)
        n = first + m
        for j in range(-(-n // 32)):
            got = c["bounds"][int(rows.case.table[0, j])].cpu().float()
            same(got[:, 0], low[32 * j:min(n, 32 * j + 32)].amin(0))
            same(got[:, 1], high[32 * j:min(n, 32 * j + 32)].amax(0))
    bare = _lib.PagedCache(d1, c["k"], c["v"], c["table"], c["kv_len"], c["new_rows"])
    old = c["bounds"].clone()
    rows.call(dict(c, cache=bare), [0], [40], dims=d1)
    assert torch.equal(c["bounds"].view(torch.uint8), old.view(torch.uint8))


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_a_run_of_them(gpu_lib, kind):
    """Prompts and then tokens of a ragged batch: rows into the pages, the attention of all new rows, within a window,
    over all and over chosen pages, on a stream of its own; then the same step from a graph, replayed among eager calls."""
    prompts, steps, W, S = [70, 1, 129], 4, 50, 3
    lens = [n + steps for n in prompts]
    rows = Rows(kind, lens, new_len=max(prompts), hq=8, hkv=2, d=128, R=16, seed=11)
    case = rows.case
    whole, held, d = list(lens), {n: list(case.held[n]) for n in "kv"}, case.dims
    c = rows.empty()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    done = [0] * 3
    with torch.cuda.stream(stream):
        for step in range(steps + 1):
            L = max(prompts) if step == 0 else 1
            new = prompts if step == 0 else [1] * 3
            dims = _lib.PagedDims.from_buffer_copy(d)
            dims.new_len = L
            q = rows.call(c, done, new, dims=dims)
            rows.check_q(q, done, new)
            done = [a + b for a, b in zip(done, new)]
            case.dims, case.lens, case.new, case.q = dims, done, new, q.cpu()
            case.held = {n: [x[:m] for x, m in zip(held[n], done)] for n in "kv"}
            if kind[0] == PD_FP32:      # the very rows that the pages hold: keys may differ by one fp32 rounding
                got = [torch.zeros(3, 2, max(done), 128, device="cuda") for _ in range(2)]
                _lib.pd_paged_read(dims, c["cache"], 0, max(done), *got)
                case.held["k"] = [h64(got[0][b, :, :done[b]].transpose(0, 1)) for b in range(3)]
            c["q"] = q
            check_window(case, *run_window(case, c, W, S, dims=dims), W, S)
            check_attn(case, *run_attn(case, c))
            if L == 1:
                idx = torch.zeros(3, 2, 3, dtype=torch.int32, device="cuda")
                ws = torch.empty(max(16, _lib.pd_paged_workspace_bytes(dims, 3, 0)), dtype=torch.uint8, device="cuda")
                _lib.pd_paged_select(dims, c["cache"], q, 3, 1, 1, idx, ws)
                check_attn(case, *run_attn(case, c, page_idx=idx), page_idx=idx.cpu())
    stream.synchronize()
    # The last step again, captured: rows written again with the same values, twice by two graphs that share a workspace.
    t = TORCH[kind[0]]
    fused = torch.stack([rows.x[b][whole[b] - 1:whole[b]] for b in range(3)]).cuda()
    o = [torch.zeros(3, 1, 8, 128, dtype=t, device="cuda") for _ in range(2)]
    lse, qo = torch.zeros(3, 8, 1, device="cuda"), torch.zeros(3, 1, 8, 128, dtype=t, device="cuda")
    ws = torch.empty(max(16, _lib.pd_paged_window_workspace_bytes(dims, W, S), _lib.pd_paged_workspace_bytes(dims, 0, 1)), dtype=torch.uint8, device="cuda")
    w = [x.cuda() for x in rows.w]

    def step(out, window):
        _lib.pd_paged_append_rope(dims, c["cache"], fused[:, :, :8], fused[:, :, 8:10], fused[:, :, 10:], *w, EPS, None, BASE, qo)
        if window:
            _lib.pd_paged_window_attn(dims, c["cache"], qo, W, S, out, lse, workspace=ws)
        else:
            _lib.pd_paged_attn(dims, c["cache"], qo, out, lse, workspace=ws)

    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            step(o[i], i == 0)
    for _ in range(3):
        for i in range(2):
            o[i].zero_()
            qo.zero_()
            graphs[i].replay()
            eager = torch.zeros_like(o[i])
            step(eager, i == 0)
            torch.cuda.synchronize()
            assert torch.equal(o[i], eager) and eager.abs().sum() > 0


def test_a_large_batch(gpu_lib):
    """Many sequences and heads: workgroups of 16 heads; one token each, then several rows."""
    for kind in KINDS[:2]:
        for L in (1, 20):
            lens = [40 + i % 30 for i in range(200)]
            rows = Rows(kind, lens, new_len=L, hq=20, hkv=5, d=64, R=16, seed=12)
            case, want = rows.case, dict(rows.case.pool)
            c = case.to_gpu()
            first = [n - L for n in lens]
            rows.check_q(rows.call(c, first, [L] * 200), first, [L] * 200)
            check_pool(case, c, want)


def test_offsets_beyond_32_bits(gpu_lib):
    """A pool of more than 2^32 bytes, and rows whose offsets pass 2^31 elements."""
    R, hkv, d = 256, 8, 128
    n_pages = (1 << 31) // (R * hkv * d) + 4
    rows = Rows(KINDS[0], [300], new_len=300, hq=8, hkv=hkv, d=d, R=R, seed=1)
    k, v = (torch.zeros(n_pages, hkv, R, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dims = _lib.PagedDims.from_buffer_copy(rows.case.dims)
    dims.n_pages = n_pages
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    kv, new = (torch.tensor([300], dtype=torch.int32, device="cuda") for _ in range(2))
    cache = _lib.PagedCache(dims, k, v, table, kv, new)
    stride = 1 << 23                                                   # elements: 300 rows are 2.5 * 2^30 elements, 5 GB
    wide = torch.empty(300 * stride, dtype=torch.bfloat16, device="cuda")
    view = wide.as_strided((1, 300, 24, d), (300 * stride, stride, d, 1))
    view.copy_(rows.x[0][None])
    q = torch.zeros(1, 300, 8, d, dtype=torch.bfloat16, device="cuda")
    _lib.pd_paged_append_rope(dims, cache, view[:, :, :8], view[:, :, 8:16], view[:, :, 16:], rows.w[0].cuda(), rows.w[1].cuda(), EPS, None, BASE, q)
    rows.check_q(q, [0], [300])
    same(k[n_pages - 2, :, :44].cpu(), rows.case.k_rows[0][256:].transpose(0, 1))
    same(v[n_pages - 1].cpu(), rows.case.v_rows[0][:256].transpose(0, 1))
