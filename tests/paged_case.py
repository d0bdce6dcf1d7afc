"""Random problems over a paged cache for the GPU tests: pages scattered over a pool, everything that no sequence holds
filled with NaN (exponent bytes with 255), and the rows as float64 for the oracle."""

import math

import numpy as np
import torch

import oracle.paged as ref
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32, PD_FP8_E4M3

TORCH = {PD_BF16: torch.bfloat16, PD_FP32: torch.float32}
HALF_STEP = {PD_BF16: 2.0 ** -8, PD_FP32: 2.0 ** -24}


def h64(t):
    return t.detach().cpu().double().numpy()


class Case:
    """lens: rows of each sequence; new: new rows of each (None: new_len each)."""

    def __init__(self, lens, new_len=1, new=None, hq=4, hkv=2, d=64, dtype=PD_BF16, cache=None, R=16, causal=1, seed=0,
                 spare=3, sigma=1.0, max_pages=None, sm_scale=0.0):
        g = torch.Generator().manual_seed(1000 + seed)
        self.g, self.lens = g, list(lens)
        self.new = list(new) if new is not None else [new_len] * len(self.lens)
        B, cache = len(self.lens), dtype if cache is None else cache
        pages = [-(-n // R) for n in self.lens]
        width = max_pages or max(1, max(pages))
        used = sum(pages)
        n_pages = used + spare
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        table = torch.full((B, width), -7, dtype=torch.int32)     # entries that no row needs
        at = 0
        for b in range(B):
            table[b, :pages[b]] = order[at:at + pages[b]]
            at += pages[b]
        self.dims = _lib.PagedDims(batch=B, new_len=new_len, n_heads_q=hq, n_heads_kv=hkv, head_dim=d, dtype=dtype,
                                   cache_dtype=cache, page_rows=R, n_pages=n_pages, max_pages=width, sm_scale=sm_scale,
                                   causal=causal)
        self.scale = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
        t = TORCH[dtype]
        rnd = lambda *s: (torch.randn(s, generator=g) * sigma).to(t)  # noqa: E731
        self.k_rows = [rnd(n, hkv, d) for n in self.lens]
        self.v_rows = [rnd(n, hkv, d) for n in self.lens]
        self.q = rnd(B, new_len, hq, d)
        self.table = table
        self.fp8 = cache == PD_FP8_E4M3
        self.place()

    # -- the pool as the sequences' rows make it
    def place(self):
        d, B = self.dims, self.dims.batch
        pool = (d.n_pages, d.n_heads_kv, d.page_rows, d.head_dim)
        self.held = {"k": [], "v": []}     # what the pages stand for, [len][H_kv][d] in float64
        self.pool = {}
        for n, rows in (("k", self.k_rows), ("v", self.v_rows)):
            if self.fp8:
                p = torch.full(pool, 0x7F, dtype=torch.uint8)
                e = torch.full(pool[:3], 255, dtype=torch.uint8)
            else:
                p = torch.full(pool, math.nan, dtype=TORCH[d.dtype])
                e = None
            for b in range(B):
                x = rows[b]
                if self.fp8:
                    val, ex = ref.quantise_ref(h64(x)) if len(x) else (np.zeros(x.shape), np.zeros(x.shape[:2], int))
                    self.held[n].append(val * 2.0 ** ex[..., None].astype(np.float64))
                    byte = torch.from_numpy(val).to(torch.float8_e4m3fn).view(torch.uint8)
                else:
                    self.held[n].append(h64(x))
                    byte = x
                for r in range(len(x)):
                    pg, sl = int(self.table[b, r // d.page_rows]), r % d.page_rows
                    p[pg, :, sl] = byte[r]
                    if e is not None:
                        e[pg, :, sl] = torch.from_numpy(ex[r] + 127).to(torch.uint8)
            self.pool[n], self.pool[n + "_exp"] = p, e
        lo = torch.full((d.n_pages, d.n_heads_kv, 2, d.head_dim), math.nan, dtype=TORCH[d.dtype])
        for b in range(B):
            for j in range(-(-self.lens[b] // d.page_rows)):
                x = self.k_rows[b][j * d.page_rows:(j + 1) * d.page_rows]
                lo[int(self.table[b, j]), :, 0] = x.amin(0)
                lo[int(self.table[b, j]), :, 1] = x.amax(0)
        self.pool["bounds"] = lo

    def to_gpu(self, device="cuda"):
        d = self.dims
        c = {k: (v.to(device) if v is not None else None) for k, v in self.pool.items()}
        c["table"], c["q"] = self.table.to(device), self.q.to(device)
        c["kv_len"] = torch.tensor(self.lens, dtype=torch.int32, device=device)
        c["new_rows"] = torch.tensor(self.new, dtype=torch.int32, device=device)
        c["cache"] = _lib.PagedCache(d, c["k"], c["v"], c["table"], c["kv_len"], c["new_rows"], c["k_exp"], c["v_exp"],
                                     c["bounds"])
        return c

    def ends(self, b):
        """Positions that the query rows (new row major, then the group's heads) of sequence b see."""
        d, G = self.dims, self.dims.n_heads_q // self.dims.n_heads_kv
        m, n = self.new[b], self.lens[b]
        return np.repeat([n - m + 1 + r if d.causal else n for r in range(m)], G)

    def rows_of(self, b, g):
        G = self.dims.n_heads_q // self.dims.n_heads_kv
        return h64(self.q[b, :self.new[b], g * G:(g + 1) * G]).reshape(-1, self.dims.head_dim)


def run_attn(case, c, page_idx=None, fill=7.0, lse=True, workspace=True, stream=None):
    d = case.dims
    o = torch.full_like(c["q"], fill)
    l = torch.full((d.batch, d.n_heads_q, d.new_len), fill, dtype=torch.float32, device=c["q"].device) if lse else None
    nb = _lib.pd_paged_workspace_bytes(d, 0 if page_idx is None else page_idx.shape[-1], 1)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device=c["q"].device) if nb and workspace else None
    _lib.pd_paged_attn(d, c["cache"], c["q"], o, l, page_idx=page_idx, workspace=ws, stream=stream)
    return o, l


def check_attn(case, o, lse, page_idx=None, fill=7.0):
    """Every row against the oracle.  Tolerance of a row, from its roundings: a score is d products summed in fp32 and
    scaled, so it is off by at most (d + 4) 2^-24 of scale * sum |q k| (twice that with the maximum's), which changes a
    weight by that factor; exp2 and the sums over N keys add 2^-21 + N 2^-24 (waves and parts add fewer); bf16
    weights are rounded by 2^-8 of themselves before they multiply V; the output is rounded once."""
    d = case.dims
    G, D = d.n_heads_q // d.n_heads_kv, d.head_dim
    o, lse = h64(o), None if lse is None else h64(lse)
    for b in range(d.batch):
        m = case.new[b]
        assert np.all(o[b, m:] == fill), "rows behind the last new one were written"
        if lse is not None:
            assert np.all(lse[b, :, m:] == fill)
        for g in range(d.n_heads_kv):
            k, v = case.held["k"][b][:, g], case.held["v"][b][:, g]
            pos = np.arange(len(k))
            if page_idx is not None:
                pages = [p for p in page_idx[b, g].tolist() if 0 <= p < d.max_pages]
                pos = np.concatenate([np.arange(p * d.page_rows, (p + 1) * d.page_rows) for p in pages] or [np.zeros(0, int)])
                pos = pos[pos < len(k)].astype(int)
                k, v = k[pos], v[pos]
            want, l, mass, spread = ref.attn_ref(case.rows_of(b, g), k, v, case.ends(b), case.scale, pos)
            got = o[b, :m, g * G:(g + 1) * G].reshape(-1, D)
            delta = (2 * (D + 4) * 2.0 ** -24 * spread + 2.0 ** -21 + len(k) * 2.0 ** -24)[:, None]
            tol = mass * (2 * delta + (2.0 ** -8 if d.dtype == PD_BF16 else 0)) + np.abs(want) * HALF_STEP[d.dtype] + 1e-37
            bad = ~(np.abs(got - want) <= tol)
            assert not bad.any(), (b, g, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], tol[bad][:3])
            if lse is not None:
                gl = lse[b, g * G:(g + 1) * G, :m].T.reshape(-1)
                tl = delta[:, 0] + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(l), l, 0)))
                ok = (gl == l) | (np.isfinite(l) & (np.abs(gl - np.where(np.isfinite(l), l, 0)) <= tl))
                assert ok.all(), (b, g, gl[~ok][:3], l[~ok][:3])
