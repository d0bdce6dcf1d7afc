"""The paged-cache calls together, as a model's layer makes them: norms and rotation of the projected rows, append, page
choice, attention; step by step, captured into graphs, on several streams; and beside the chunk path's own calls."""

import math

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged_case import HALF_STEP, Case, check_attn, h64, run_attn
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3, Dims

pytestmark = pytest.mark.gpu
BASE, EPS = 5e5, 1e-6


class Layer:
    """One layer's cache and buffers for B sequences of at most `most` rows, prompts appended first."""

    def __init__(self, prompts, most, hq=4, hkv=2, d=64, dtype=PD_BF16, cache=PD_FP8_E4M3, R=16, top_k=3, seed=0):
        t = {PD_BF16: torch.bfloat16, PD_FP32: torch.float32}
        B, pages, g = len(prompts), -(-most // R), torch.Generator().manual_seed(seed)
        self.g, self.hq, self.hkv, self.d, self.top_k, self.t, self.B = g, hq, hkv, d, top_k, t[dtype], B
        self.dims = _lib.PagedDims(batch=B, new_len=1, n_heads_q=hq, n_heads_kv=hkv, head_dim=d, dtype=dtype,
                                   cache_dtype=cache, page_rows=R, n_pages=B * pages, max_pages=pages, causal=1)
        self.table = torch.randperm(B * pages, generator=g).to(torch.int32).view(B, pages).cuda()
        ct = torch.float8_e4m3fn if cache == PD_FP8_E4M3 else self.t
        mk = lambda *s, dt: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
        self.k, self.v = (mk(B * pages, hkv, R, d, dt=ct) for _ in range(2))
        ex = [mk(B * pages, hkv, R, dt=torch.uint8) if cache == PD_FP8_E4M3 else None for _ in range(2)]
        self.bounds = mk(B * pages, hkv, 2, d, dt=self.t)
        self.kv_len = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        self.new_rows = self.kv_len.clone()
        self.cache = _lib.PagedCache(self.dims, self.k, self.v, self.table, self.kv_len, self.new_rows, ex[0], ex[1], self.bounds)
        self.w = [(1 + 0.2 * torch.randn(d, generator=g)).to(self.t).cuda() for _ in range(2)]
        self.idx = torch.zeros(B, hkv, top_k, dtype=torch.int32, device="cuda")
        self.ws = [torch.empty(max(16, _lib.pd_paged_workspace_bytes(self.dims, top_k, i)), dtype=torch.uint8, device="cuda")
                   for i in (0, 1)]
        self.rows = [[[], []] for _ in range(B)]       # what the cache holds, in float64
        self.prompts = prompts

    def projected(self, L):
        return torch.randn(self.B, L, self.hq + 2 * self.hkv, self.d, generator=self.g).to(self.t)

    def step(self, x, pos, L, stream=None):
        """x [B, L, H_q + 2 H_kv, d] on the GPU -> o, lse over the chosen pages; L = 1 or a prompt (attends to all pages)."""
        d = _lib.PagedDims.from_buffer_copy(self.dims)
        d.new_len = L
        T, hq, hkv = self.B * L, self.hq, self.hkv
        flat = x.view(T, hq + 2 * hkv, self.d)
        q, k = torch.empty(T, hq, self.d, dtype=self.t, device="cuda"), torch.empty(T, hkv, self.d, dtype=self.t, device="cuda")
        _lib.pd_qk_norm_rope(flat[:, :hq], flat[:, hq:hq + hkv], self.w[0], self.w[1], EPS, pos, BASE, q, k, stream=stream)
        q, k = q.view(self.B, L, hq, self.d), k.view(self.B, L, hkv, self.d)
        _lib.pd_paged_append(d, self.cache, k, x[:, :, hq + hkv:], stream=stream)
        o, lse = torch.zeros_like(q), torch.zeros(self.B, hq, L, device="cuda")
        if L == 1:
            _lib.pd_paged_select(d, self.cache, q, self.top_k, 1, 1, self.idx, self.ws[0], stream=stream)
            _lib.pd_paged_attn(d, self.cache, q, o, lse, page_idx=self.idx, workspace=self.ws[1], stream=stream)
        else:
            n = _lib.pd_paged_workspace_bytes(d, 0, 1)
            _lib.pd_paged_attn(d, self.cache, q, o, lse, workspace=torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"),
                               stream=stream)
        return q, k, o, lse


@pytest.mark.parametrize("dtype,cache", [(PD_BF16, PD_FP8_E4M3), (PD_BF16, PD_BF16), (PD_FP32, PD_FP32)])
def test_prompt_and_steps(gpu_lib, dtype, cache):
    """A ragged batch's prompts and five tokens each.  The queries and keys of a step are held to the norm's bar by its
    own tests; here the pages and the attention are checked on the very rows that the calls wrote."""
    prompts = [70, 1, 129]
    y = Layer(prompts, 160, dtype=dtype, cache=cache, seed=4)
    hq, hkv, G = y.hq, y.hkv, y.hq // y.hkv
    lens = [0] * y.B
    for step in range(6):
        L = max(prompts) if step == 0 else 1
        new = prompts if step == 0 else [1] * y.B
        lens = [a + b for a, b in zip(lens, new)]
        y.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        y.new_rows.copy_(torch.tensor(new, dtype=torch.int32))
        pos = torch.tensor([[lens[b] - new[b] + r for r in range(L)] for b in range(y.B)], dtype=torch.int32).view(-1)
        x = y.projected(L)
        q, k, o, lse = y.step(x.cuda(), pos.cuda(), L)
        torch.cuda.synchronize()
        want_q = ref.qk_norm_rope_ref(h64(x.view(-1, hq + 2 * hkv, y.d)[:, :hq]), h64(y.w[0]), EPS, pos.numpy(), BASE)
        np.testing.assert_allclose(h64(q).reshape(want_q.shape), want_q, atol=8 * 2.0 ** -8)   # |q| < 8: one rounding
        case = Case.__new__(Case)
        case.dims = _lib.PagedDims.from_buffer_copy(y.dims)
        case.dims.new_len = L
        case.lens, case.new, case.q, case.scale = lens, new, q.cpu(), 1 / math.sqrt(y.d)
        for b in range(y.B):
            for i, rows in enumerate((h64(k)[b, :new[b]], h64(x)[b, :new[b], hq + hkv:])):
                if cache == PD_FP8_E4M3:
                    val, e = ref.quantise_ref(rows)
                    rows = val * 2.0 ** e[..., None].astype(np.float64)
                y.rows[b][i].append(rows)
        case.held = {n: [np.concatenate(y.rows[b][i]) for b in range(y.B)] for i, n in enumerate("kv")}
        if L == 1:
            idx, bounds, table = y.idx.cpu(), h64(y.bounds), y.table.cpu().long().numpy()
            for b in range(y.B):
                pages = -(-lens[b] // y.dims.page_rows)
                for g in range(hkv):
                    lo, hi = (bounds[table[b, :pages], g, i] for i in range(2))
                    s = ref.page_scores_ref(h64(q)[b, 0, g * G:(g + 1) * G], lo, hi)
                    best = ref.select_ref(s, y.top_k, 1, 1)
                    assert idx[b, g].tolist() == best + [-1] * (y.top_k - len(best))
            check_attn(case, o, lse, page_idx=idx, fill=0.0)
        else:
            check_attn(case, o, lse, fill=0.0)


def test_graphs_replayed_among_eager_work(gpu_lib):
    """A step captured twice (two graphs that share the layer's workspaces), replayed in turn with eager steps and
    synchronisations between: the bits of the eager step every time."""
    y = Layer([300, 41, 7], 400, hq=8, hkv=2, d=128, R=16, top_k=4, seed=5)
    L = max(y.prompts)
    pos = torch.arange(L, dtype=torch.int32).repeat(y.B).cuda()
    y.step(y.projected(L).cuda(), pos, L)
    y.kv_len.add_(1)
    y.new_rows.fill_(1)
    steps = [(y.projected(1).cuda(), (y.kv_len - 1).clone()) for _ in range(3)]
    want = []
    for x, p in steps:
        q, k, o, lse = y.step(x, p, 1)
        torch.cuda.synchronize()
        want.append((y.idx.clone(), o.clone(), lse.clone()))
    # Every step writes the same position, whose row and page bounds the later ones widen: once more from a settled state.
    want = []
    for x, p in steps:
        q, k, o, lse = y.step(x, p, 1)
        torch.cuda.synchronize()
        want.append((y.idx.clone(), o.clone(), lse.clone()))
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for x, p in steps[:2]:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                outs.append(y.step(x, p, 1))
        graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(4):
        x, p = steps[2]
        _, _, o, lse = y.step(x, p, 1)
        torch.cuda.synchronize()
        for a, b in zip((y.idx, o, lse), want[2]):
            assert torch.equal(a, b)
        for i in (turn % 2, 1 - turn % 2):
            graphs[i].replay()
            torch.cuda.synchronize()
            for a, b in zip((y.idx, outs[i][2], outs[i][3]), want[i]):
                assert torch.equal(a, b), (turn, i)


def test_streams(gpu_lib):
    """Calls on three streams at once, each with its own cache, workspace and outputs, give the bits of a run in turn."""
    layers = [Layer([500 + 100 * i, 33], 900, hq=4, hkv=2, d=128, top_k=5, seed=i) for i in range(3)]
    work = []
    for y in layers:
        L = max(y.prompts)
        work.append((y, y.projected(L).cuda(), torch.arange(L, dtype=torch.int32).repeat(y.B).cuda(), L, y.projected(1).cuda()))

    def go(y, x, pos, L, tok, stream):
        y.kv_len.copy_(torch.tensor(y.prompts, dtype=torch.int32, device="cuda"))
        y.new_rows.copy_(y.kv_len)
        a = y.step(x, pos, L, stream)[2]
        y.kv_len.add_(1)
        y.new_rows.fill_(1)
        b = y.step(tok, y.kv_len - 1, 1, stream)[2]
        return a, b

    want = []
    for w in work:
        want.append([t.clone() for t in go(*w, torch.cuda.current_stream())])
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream() for _ in layers]
    for w, s in zip(work, streams):
        with torch.cuda.stream(s):
            got.append(go(*w, s))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("cache", [PD_BF16, PD_FP8_E4M3])
def test_read_back_feeds_the_compact_decode(gpu_lib, cache):
    """A block of 32 rows over 200 cached ones: pd_paged_attn without a causal mask, and pd_paged_read into the prefix of
    pd_sparse_decode_attn_compact, which holds the block's own rows beside it.  With a bf16 cache both are the same
    attention; an 8-bit cache also holds the block's rows in 8 bits, so the block's rows are read back for the compact
    call too."""
    B, n, L, hq, hkv, d = 2, 200, 32, 8, 2, 128
    case = Case([n + L] * B, new_len=L, hq=hq, hkv=hkv, d=d, cache=cache, R=64, causal=0, seed=9)
    c = case.to_gpu()
    o, lse = run_attn(case, c)
    check_attn(case, o, lse)
    pre = [torch.empty(B, hkv, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    own = [torch.empty(B, hkv, L, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(case.dims, c["cache"], 0, n, *pre)
    _lib.pd_paged_read(case.dims, c["cache"], n, L, *own)
    own = [t.transpose(1, 2).contiguous() for t in own]
    dims = Dims(B, 1, 16, 1, 0, L, hq, hkv, d, PD_BF16)
    od, ld = torch.empty_like(c["q"]), torch.empty(B, hq, L, device="cuda")
    ws = torch.empty(max(16, _lib.pd_compact_workspace_bytes(dims, n)), dtype=torch.uint8, device="cuda")
    _lib.pd_sparse_decode_attn_compact(dims, n, c["q"], *own, *pre, None, None, 0, od, ld, 0, ws)
    torch.cuda.synchronize()
    check_attn(case, od, None)           # the same rows within the same bar
    # its LSE is that of the rounded weights: within log(1 + 2^-8)
    assert (lse - ld).abs().max().item() <= math.log1p(2.0 ** -8) + 1e-3


def test_binding_refuses_what_does_not_fit(gpu_lib):
    case = Case([40, 20], hq=4, hkv=2, d=64, R=16, seed=1)
    c, d = case.to_gpu(), case.dims
    ok = dict(k_pages=c["k"], v_pages=c["v"], page_table=c["table"], kv_len=c["kv_len"])
    for bad in (dict(k_pages=c["k"][:-1]), dict(v_pages=c["v"].float()), dict(page_table=c["table"].long()),
                dict(page_table=c["table"][:1]), dict(kv_len=c["kv_len"].cpu()), dict(new_rows=c["kv_len"][:1]),
                dict(k_exp=torch.zeros(1)), dict(k_bounds=c["bounds"][:, :, :1])):
        with pytest.raises(ValueError):
            _lib.PagedCache(d, **{**ok, **bad})
    o = torch.zeros_like(c["q"])
    for q, out, lse in ((c["q"][:1], o, None), (c["q"].float(), o, None), (c["q"], o[:, :, :1], None),
                        (c["q"], o, torch.zeros(2, 4, 2, device="cuda"))):
        with pytest.raises(ValueError):
            _lib.pd_paged_attn(d, c["cache"], q, out, lse)
    other = _lib.PagedDims.from_buffer_copy(d)
    other.n_pages += 1
    with pytest.raises(ValueError):
        _lib.pd_paged_attn(other, c["cache"], c["q"], o)
    x = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        _lib.pd_paged_append(d, c["cache"], x, x.float())
    with pytest.raises(ValueError):
        _lib.pd_paged_append(d, c["cache"], x[:1], x)
    with pytest.raises(_lib.PdError):
        _lib.pd_paged_read(d, c["cache"], 0, 49, *(torch.zeros(2, 2, 49, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    torch.cuda.synchronize()


def test_no_launch_beside_the_current_device(gpu_lib):
    with pytest.raises(ValueError, match="current"):
        _lib._launch_stream(None, torch.cuda.current_device() + 1)


def test_grids_beyond_one_dimension(gpu_lib):
    """More than 2^20 workgroups in every launch: 5 million rows of one head normalised and rotated, and a token of
    40000 sequences of 32 heads, all with the same page contents, appended, chosen from, attended to and read back."""
    T, d = 5_000_000, 64
    x = torch.randn(T, 1, d, device="cuda").to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    _lib.pd_qk_norm_rope(x, None, None, None, 0.0, pos, 1e4, y, None)
    at = torch.tensor([0, 1, 4_194_303, 4_194_304, T - 1], device="cuda")
    want = ref.qk_norm_rope_ref(h64(x[at]), None, 0, h64(pos[at]), 1e4)
    assert np.all(np.abs(h64(y[at]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * 8)
    assert torch.allclose(y.float().norm(dim=-1), x.float().norm(dim=-1), rtol=2.0 ** -7)    # turned, not stretched
    del x, y
    B, H, R = 40000, 32, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    row = lambda h: torch.randn(1, 1, h, d, generator=g, device="cuda").to(torch.bfloat16).expand(B, 1, h, d).contiguous()  # noqa: E731
    dims = _lib.PagedDims(batch=B, new_len=1, n_heads_q=H, n_heads_kv=H, head_dim=d, dtype=PD_BF16, cache_dtype=PD_BF16,
                          page_rows=R, n_pages=B, max_pages=1, causal=1)
    k, v = (torch.zeros(B, H, R, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    bounds = torch.zeros(B, H, 2, d, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(B - 1, -1, -1, dtype=torch.int32, device="cuda").view(B, 1)
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache = _lib.PagedCache(dims, k, v, table, kv_len, k_bounds=bounds)
    rows = []
    for _ in range(3):
        kv_len.add_(1)
        rows.append((row(H), row(H)))
        _lib.pd_paged_append(dims, cache, *rows[-1])
    assert torch.equal(k, k[:1].expand_as(k)) and torch.equal(bounds, bounds[:1].expand_as(bounds))
    assert torch.equal(v[0, :, :3], torch.cat([r[1][0] for r in rows]).transpose(0, 1))
    q, idx = row(H), torch.empty(B, H, 1, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(_lib.pd_paged_workspace_bytes(dims, 1, 0), 16), dtype=torch.uint8, device="cuda")
    _lib.pd_paged_select(dims, cache, q, 1, 0, 0, idx, ws)
    assert torch.all(idx == 0)
    assert _lib.pd_paged_workspace_bytes(dims, 1, 1) == 0
    o, lse = torch.empty_like(q), torch.empty(B, H, 1, device="cuda")
    for sel in (None, idx):
        o.zero_()
        _lib.pd_paged_attn(dims, cache, q, o, lse, page_idx=sel)
        assert torch.equal(o, o[:1].expand_as(o)) and torch.equal(lse, lse[:1].expand_as(lse))
        for h in (0, 17, 31):
            want, l, mass, _ = ref.attn_ref(h64(q[0, :, h]), h64(k[0, h, :3]), h64(v[0, h, :3]), [3], d ** -0.5)
            assert np.all(np.abs(h64(o[0, :, h]) - want) <= 2.0 ** -8 * (mass + np.abs(want)) + 2.0 ** -17 * mass)
            assert abs(lse[0, h, 0].item() - l[0]) < 1e-5
    out = [torch.empty(B, H, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    _lib.pd_paged_read(dims, cache, 1, 2, *out)
    assert torch.equal(out[0], out[0][:1].expand_as(out[0])) and torch.equal(out[0][0], k[0, :, 1:3])


def test_streams_over_spoilt_caches(gpu_lib):
    """Three layers at once on streams of their own, over pages, bounds, lists and workspaces that hold nothing but NaN,
    255 and -1 before: a call that ran ahead of the one whose results it reads would show it."""
    def fresh():
        out = []
        for i in range(3):
            y = Layer([500 + 100 * i, 33], 900, hq=4, hkv=2, d=128, top_k=5, seed=i)
            for t in (y.k, y.v, *y.cache.tensors[2:4]):
                t.view(torch.uint8).fill_(255)
            y.bounds.fill_(math.nan)
            y.idx.fill_(-1)
            for w in y.ws:
                w.fill_(255)
            L = max(y.prompts)
            out.append((y, y.projected(L).cuda(), torch.arange(L, dtype=torch.int32).repeat(y.B).cuda(), L,
                        [y.projected(1).cuda() for _ in range(4)]))
        torch.cuda.synchronize()
        return out

    def go(y, x, pos, L, tokens, stream):
        y.kv_len.copy_(torch.tensor(y.prompts, dtype=torch.int32, device="cuda"))
        y.new_rows.copy_(y.kv_len)
        outs = [y.step(x, pos, L, stream)[2:]]
        y.new_rows.fill_(1)
        for tok in tokens:
            y.kv_len.add_(1)
            outs.append((*y.step(tok, y.kv_len - 1, 1, stream)[2:], y.idx.clone()))
        return outs

    want = []
    for w in fresh():
        want.append(go(*w, torch.cuda.current_stream()))
        torch.cuda.synchronize()
    got, layers, streams = [], fresh(), [torch.cuda.Stream() for _ in range(3)]
    for w, s in zip(layers, streams):
        with torch.cuda.stream(s):
            got.append(go(*w, s))
    torch.cuda.synchronize()
    for layer in zip(got, want):
        for step in zip(*layer):
            for a, b in zip(*step):
                assert torch.equal(a, b)
    assert all(torch.isfinite(t).all() for outs in want for step in outs for t in step[:1])
