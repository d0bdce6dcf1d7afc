"""The operators around the paged key/value cache, in plain form and through the binding, and the cases that they
are timed on.

* ``norm``   -- pd_qk_norm_rope: RMS norms of the query and key heads and their rotary positions, one pass;
* ``append`` -- pd_paged_append: new rows into the pages, quantised to 8 bits where the cache is, with the
  per-channel bounds of each page's keys;
* ``read``   -- pd_paged_read: rows of the pages back into contiguous buffers;
* ``attn``   -- pd_paged_attn: attention of one or a few new rows over the pages;
* ``sparse`` -- pd_paged_select, then pd_paged_attn over the pages that it chose.

A cache of 8 bits holds a head's row as E4M3 values times a power of two, whose exponent e is kept as the byte
e + 127: the least e with max|x| <= 448 * 2^e, within -100..120.
"""

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "fp8": 1}
_EPS = 1e-6
_BASE = 5e5

_DEFAULT = {"op": "attn", "dtype": "bf16", "cache": "bf16", "batch": 1, "new_len": 1, "kv_len": 8192, "ragged": False,
            "heads_q": 32, "heads_kv": 32, "head_dim": 128, "page_rows": 64, "causal": True, "bounds": True,
            "top_k": 0, "first": 1, "last": 2}


def _case(name=None, **kw):
    c = dict(_DEFAULT, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One token of one request, 7 query heads per key head: the latency of a launch.
        _case("norm_token_gqa", op="norm", new_len=1, heads_q=28, heads_kv=4),
        # The tokens of an odd batch of short prompts, in full precision, d = 64.
        _case("norm_ragged_fp32_d64", op="norm", dtype="fp32", new_len=777, heads_q=12, heads_kv=4, head_dim=64),
        # A whole 32K prompt ahead of its chunk prefill: the largest call.
        _case("norm_prompt_32k", op="norm", new_len=32768),
        # A decoding step of eight requests of different lengths, 8-bit cache.
        _case("append_token_fp8", op="append", cache="fp8", batch=8, ragged=True, heads_q=28, heads_kv=4),
        # Prompts of four requests, of odd lengths up to 4161 rows, into an 8-bit cache.
        _case("append_prompt_fp8", op="append", cache="fp8", batch=4, new_len=4161, kv_len=4161, ragged=True),
        # The kept rows of four requests back as bf16, as the prefix of a block decode.
        _case("read_fp8", op="read", cache="fp8", batch=4, kv_len=8192, ragged=True, heads_kv=8),
        # The next token of one 8K request: few workgroups, the split and the join count.
        _case("attn_token_8k_gqa", heads_q=28, heads_kv=4),
        # The next tokens of eight 32K requests with as many key heads as query heads: the largest call.
        _case("attn_token_32k_b8", batch=8, kv_len=32768),
        # A serving batch of 64 requests of 512 to 32K rows, small pages, 8-bit cache, 4 query heads per key head.
        _case("attn_serving_fp8", cache="fp8", batch=64, kv_len=32768, ragged=True, heads_kv=8, page_rows=16),
        # A denoising block of 32 rows that see each other, in full precision, d = 64.
        _case("attn_block32_fp32", dtype="fp32", cache="fp32", batch=2, new_len=32, kv_len=1000, ragged=True,
              heads_q=8, heads_kv=4, head_dim=64, page_rows=32, causal=False),
        # The next tokens of eight 32K requests, 32 of 512 pages for each key head.
        _case("sparse_32k_b8", op="sparse", batch=8, kv_len=32768, top_k=32),
        # Two 128K requests, 8-bit cache, 64 of 2048 pages for each group of four query heads.
        _case("sparse_128k_fp8", op="sparse", cache="fp8", batch=2, kv_len=131072, heads_kv=8, top_k=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["norm", "append", "read", "attn", "attn", "attn", "sparse", "sparse"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        hkv = rng.choice([1, 2, 4, 8, 32])
        hq = hkv * (rng.choice([1, 2, 4, 7, 8]) if hkv < 32 else 1)
        ragged = rng.random() < 0.6
        case = _case(op=op, dtype=dtype, cache=rng.choice([dtype, "fp8"]) if dtype == "bf16" else dtype,
                     batch=_log(rng, 1, 64), kv_len=_log(rng, 33, 131072), ragged=ragged, heads_q=hq, heads_kv=hkv,
                     head_dim=rng.choice([64, 128, 128]), page_rows=rng.choice([16, 32, 64, 64, 128, 256]),
                     causal=rng.random() < 0.7)
        if op == "norm":
            case.update(batch=1, new_len=_log(rng, 1, 32768))
        elif op == "append":
            case.update(new_len=rng.choice([1, 1, _log(rng, 1, case["kv_len"])]), bounds=rng.random() < 0.7)
        elif op != "read":
            case.update(new_len=rng.choice([1, 1, 1, rng.randint(2, 33)]))
        if op == "sparse":
            pages = -(-case["kv_len"] // case["page_rows"])
            if pages < 8:
                continue
            case.update(top_k=rng.randint(4, max(4, min(128, pages // 2))), first=rng.randint(0, 2),
                        last=rng.randint(0, 2))
        w, rows = work(case), sum(_lengths(case))
        # A plain form holds every key of the batch in 32 bits.
        if w["bytes"] <= largest and w["flops"] <= 4e10 and rows * hkv * case["head_dim"] <= 1 << 30:
            return case


# ------------------------------------------------------------------------------------------- sizes

def _lengths(c):
    """Rows of each sequence, the new ones included: spread evenly up to kv_len in a scattered order, or all kv_len."""
    B, n = c["batch"], c["kv_len"]
    if not c["ragged"]:
        return [n] * B
    least = 1 if c["op"] == "append" else c["new_len"]   # prompts may be shorter than the places for new rows
    step = 37 if B % 37 else 1
    return [max(least, n * (b * step % B + 1) // B) for b in range(B)]


def _new_rows(c):
    return [min(c["new_len"], n) for n in _lengths(c)]


def _pages(c, n):
    return -(-n // c["page_rows"])


def work(case):
    """Bytes and operations that one pass cannot do without: inputs read once, outputs written once."""
    c = case
    eb, cb, d, hq, hkv = _BYTES[c["dtype"]], _BYTES[c["cache"]], c["head_dim"], c["heads_q"], c["heads_kv"]
    row = d * cb + (1 if c["cache"] == "fp8" else 0)   # one head's row in the cache
    lens, new = _lengths(c), _new_rows(c)
    if c["op"] == "norm":
        n = c["new_len"] * (hq + hkv) * d
        return {"bytes": 2 * n * eb + 4 * c["new_len"], "flops": 8 * n}
    if c["op"] == "append":
        n = sum(new) * hkv * 2
        touched = sum(_pages(c, s) - (s - m) // c["page_rows"] for s, m in zip(lens, new))
        return {"bytes": n * (d * eb + row) + (touched * hkv * 2 * d * eb if c["bounds"] else 0), "flops": 4 * n * d}
    if c["op"] == "read":
        n = sum(lens) * hkv * 2
        return {"bytes": n * (d * eb + row), "flops": n * d}
    by = fl = 0
    for s, m in zip(lens, new):
        rows, pages = s, _pages(c, s)
        if c["op"] == "sparse":
            rows = min(s, c["top_k"] * c["page_rows"])
            by += pages * hkv * 2 * d * eb + min(pages, c["top_k"]) * hkv * 4
            fl += 2 * pages * hq * m * d
        by += rows * hkv * 2 * row + m * hq * (2 * d * eb + 4)
        fl += 4 * rows * hq * m * d
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _exponent(x):
    """The exponent of a row's power of two, from its largest magnitude (over the last dimension)."""
    m, e = torch.frexp(x.abs().amax(-1))          # m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(m == 0, -100, e).clamp(-100, 120)


def _quantised(x):
    e = _exponent(x)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    c, g = case, _gen(seed)
    t, d, hq, hkv, R, B = _TYPES[c["dtype"]], c["head_dim"], c["heads_q"], c["heads_kv"], c["page_rows"], c["batch"]
    s = {"case": c}
    if c["op"] == "norm":
        # The rows of a fused projection [q | k | v], positions of several requests one after another.
        T = c["new_len"]
        fused = (_normal(g, T, hq + 2 * hkv, d) * 1.5).to(t)
        s["q"], s["k"] = fused[:, :hq], fused[:, hq:hq + hkv]
        s["w_q"], s["w_k"] = ((1 + 0.2 * _normal(g, d)).to(t) for _ in range(2))
        s["pos"] = ((torch.arange(T, device="cuda") * 3 + int(seed) % 1000) % 131072).to(torch.int32)
        s["q_out"], s["k_out"] = torch.empty((T, hq, d), dtype=t, device="cuda"), torch.empty((T, hkv, d), dtype=t, device="cuda")
        return s
    lens, new = _lengths(c), _new_rows(c)
    width = _pages(c, max(lens))
    used = sum(_pages(c, n) for n in lens)
    # The pages lie scattered in the pool; its last page is in no table.
    order = torch.randperm(used, generator=g, device="cuda").to(torch.int32)
    s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["new_rows"] = torch.tensor(new, dtype=torch.int32, device="cuda")
    counts = torch.tensor([_pages(c, n) for n in lens], device="cuda")
    at = torch.arange(width, device="cuda")
    starts = torch.cumsum(counts, 0) - counts
    inside = at[None] < counts[:, None]
    s["table"] = torch.where(inside, order[(starts[:, None] + at[None]).clamp(max=used - 1)], 0).to(torch.int32).contiguous()
    pool = (used + 1, hkv, R, d)
    k, v = (_normal(g, *pool) for _ in range(2))
    k *= torch.exp(0.3 * _normal(g, used + 1, hkv, R, 1))      # key norms with a heavy tail
    if c["op"] == "sparse":
        # Some pages hold what the query asks for: a direction of each key head.
        u = _normal(g, hkv, d)
        k += 2.0 * (torch.rand((used + 1, hkv), generator=g, device="cuda") < 0.05)[..., None, None] * u[None, :, None] * (d ** -0.25)
    k, v = k.to(t), v.to(t)
    if c["op"] in ("append", "sparse") and c["bounds"]:
        # Bounds of the rows that the sequences hold.
        page_len = torch.full((used + 1,), R, device="cuda")
        page_len[order[(starts + counts - 1)].long()] = s["kv_len"].long() - (counts - 1) * R
        hidden = (torch.arange(R, device="cuda")[None] >= page_len[:, None])[:, None, :, None]
        s["bounds"] = torch.stack([k.masked_fill(hidden, math.inf).amin(2), k.masked_fill(hidden, -math.inf).amax(2)], 2).contiguous()
    if c["cache"] == "fp8":
        s["k"], s["k_exp"] = _quantised(k.float())
        s["v"], s["v_exp"] = _quantised(v.float())
    else:
        s["k"], s["v"] = k, v
    if c["op"] == "append":
        fused = _normal(g, B, c["new_len"], 2 * hkv, d).to(t)
        s["k_new"], s["v_new"] = fused[:, :, :hkv], fused[:, :, hkv:]
    elif c["op"] == "read":
        s["k_out"], s["v_out"] = (torch.zeros((B, hkv, max(lens), d), dtype=t, device="cuda") for _ in range(2))
    else:
        q = _normal(g, B, c["new_len"], hq, d)
        if c["op"] == "sparse":
            q += 0.5 * u.repeat_interleave(hq // hkv, 0)
        s["q"] = q.to(t)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, hq, c["new_len"]), device="cuda")
        if c["op"] == "sparse":
            s["page_idx"] = torch.zeros((B, hkv, c["top_k"]), dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------- the passes

def run(state):
    if own:
        return _own(state)
    return {"norm": _norm, "append": _append, "read": _read, "attn": _attn, "sparse": _sparse}[state["case"]["op"]](state)


def _plan(s):
    """Sizes, cache descriptor and workspaces, as a program keeps them."""
    from paper_2606_10537_amd import _lib
    c = s["case"]
    kinds = {"bf16": _lib.PD_BF16, "fp32": _lib.PD_FP32, "fp8": _lib.PD_FP8_E4M3}
    dims = _lib.PagedDims(batch=c["batch"], new_len=c["new_len"], n_heads_q=c["heads_q"], n_heads_kv=c["heads_kv"],
                          head_dim=c["head_dim"], dtype=kinds[c["dtype"]], cache_dtype=kinds[c["cache"]],
                          page_rows=c["page_rows"], n_pages=s["k"].shape[0], max_pages=s["table"].shape[1],
                          causal=int(c["causal"]))
    cache = _lib.PagedCache(dims, s["k"], s["v"], s["table"], s["kv_len"], new_rows=s["new_rows"], k_exp=s.get("k_exp"),
                            v_exp=s.get("v_exp"), k_bounds=s.get("bounds"))
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
          for n in (_lib.pd_paged_workspace_bytes(dims, c["top_k"], which) for which in (0, 1))]
    return dims, cache, ws


def _own(s):
    from paper_2606_10537_amd import _lib
    c = s["case"]
    if c["op"] == "norm":
        _lib.pd_qk_norm_rope(s["q"], s["k"], s["w_q"], s["w_k"], _EPS, s["pos"], _BASE, s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if "plan" not in s:
        s["plan"] = _plan(s)
    dims, cache, ws = s["plan"]
    if c["op"] == "append":
        _lib.pd_paged_append(dims, cache, s["k_new"], s["v_new"])
        return _pool(s)
    if c["op"] == "read":
        _lib.pd_paged_read(dims, cache, 0, s["k_out"].shape[2], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    if c["op"] == "attn":
        _lib.pd_paged_attn(dims, cache, s["q"], s["o"], s["lse"], workspace=ws[1])
        return s["o"], s["lse"]
    _lib.pd_paged_select(dims, cache, s["q"], c["top_k"], c["first"], c["last"], s["page_idx"], ws[0])
    _lib.pd_paged_attn(dims, cache, s["q"], s["o"], s["lse"], page_idx=s["page_idx"], workspace=ws[1])
    return s["page_idx"], s["o"], s["lse"]


def _pool(s):
    """What an append leaves in the pages of the sequences (the spare page takes the plain form's padding rows)."""
    return {n: s[n][:-1] for n in ("k", "v", "k_exp", "v_exp", "bounds") if n in s}


def _norm(s):
    def one(x, w, out):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.float()
        a, b = y.chunk(2, -1)
        out.copy_(torch.cat([a * cos - b * sin, b * cos + a * sin], -1))
        return out

    half = s["q"].shape[-1] // 2
    freq = _BASE ** (torch.arange(half, device="cuda", dtype=torch.float64) / -half)
    angle = s["pos"].double()[:, None, None] * freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    return one(s["q"], s["w_q"], s["q_out"]), one(s["k"], s["w_k"], s["k_out"])


def _append(s):
    c = s["case"]
    R, spare = c["page_rows"], s["k"].shape[0] - 1
    r = torch.arange(c["new_len"], device="cuda")
    real = r[None] < s["new_rows"][:, None]
    pos = (s["kv_len"] - s["new_rows"])[:, None] + r[None]
    page = torch.where(real, s["table"].gather(1, (pos // R).clamp(0, s["table"].shape[1] - 1).long()), spare).long().reshape(-1)
    slot = torch.where(real, pos % R, 0).long().reshape(-1)
    for name in ("k", "v"):
        x = s[name + "_new"].flatten(0, 1)
        if c["cache"] == "fp8":
            x, e = _quantised(x.float())
            s[name + "_exp"][page, :, slot] = e
            s[name].view(torch.uint8)[page, :, slot] = x.view(torch.uint8)
        else:
            s[name][page, :, slot] = x
    if c["bounds"]:
        x, old = s["k_new"].flatten(0, 1).float(), s["bounds"].float()
        low = torch.full_like(old[:, :, 0], math.inf).index_reduce_(0, page, x, "amin")
        high = torch.full_like(old[:, :, 1], -math.inf).index_reduce_(0, page, x, "amax")
        fresh = torch.zeros(spare + 1, device="cuda").index_put_((page,), (slot == 0).float(), accumulate=True) > 0
        fresh = fresh[:, None, None]   # a page whose first row is written begins anew
        low = torch.where(fresh, low, torch.minimum(old[:, :, 0], low))
        high = torch.where(fresh, high, torch.maximum(old[:, :, 1], high))
        s["bounds"].copy_(torch.stack([low, high], 2))
    return _pool(s)


def _rows(s, name, page, head):
    """Rows of the pages as 32-bit values, dequantised where the cache is in 8 bits."""
    x = s[name][page, head]
    if name + "_exp" in s:
        x = torch.ldexp(x.float(), (s[name + "_exp"][page, head].int() - 127)[..., None])
    return x.float()


def _read(s):
    c = s["case"]
    n, R = s["k_out"].shape[2], c["page_rows"]
    pos = torch.arange(n, device="cuda")
    page = s["table"][:, pos // R].long()[:, None]
    head = torch.arange(c["heads_kv"], device="cuda")[None, :, None]
    valid = (pos[None] < s["kv_len"][:, None])[:, None, :, None]
    for name in ("k", "v"):
        x = s[name][page, head, pos % R]
        if c["cache"] == "fp8":
            x = torch.ldexp(x.float(), (s[name + "_exp"][page, head, pos % R].int() - 127)[..., None])
        out = s[name + "_out"]
        out.copy_(torch.where(valid, x.to(out.dtype), out))
    return s["k_out"], s["v_out"]


def _attend(s, idx):
    """Attention over the rows of the logical pages idx [B][H_kv][n] (-1: none)."""
    c = s["case"]
    B, L, hq, d, hkv, R = c["batch"], c["new_len"], c["heads_q"], c["head_dim"], c["heads_kv"], c["page_rows"]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    phys = s["table"][:, None].expand(B, hkv, -1).gather(2, idx.clamp(min=0).long()).long()
    k, v = (_rows(s, n, phys, head).flatten(2, 3) for n in ("k", "v"))
    pos = (idx[..., None] * R + torch.arange(R, device="cuda")).masked_fill(idx[..., None] < 0, 1 << 30).flatten(2, 3)
    q = s["q"].float().view(B, L, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [B][H_kv][L * G][d]
    row = torch.arange(L, device="cuda")[None]
    end = s["kv_len"][:, None] - (s["new_rows"][:, None] - 1 - row if c["causal"] else 0) + 0 * row
    end = end.repeat_interleave(hq // hkv, 1)[:, None, :, None]
    unseen = pos[:, :, None] >= end
    w = ((q @ k.transpose(2, 3)) * d ** -0.5).masked_fill_(unseen, -math.inf)
    del k
    top = w.amax(-1, keepdim=True).clamp(min=-1e30)
    w = torch.exp_(w.sub_(top))
    total = w.sum(-1, keepdim=True)
    v.masked_fill_((pos >= s["kv_len"][:, None, None])[..., None], 0)
    o = (w @ v) / torch.where(total > 0, total, 1)
    lse = (top + torch.log(total)).squeeze(-1)
    real = (row < s["new_rows"][:, None])
    o = o.view(B, hkv, L, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, L, hq, d)
    lse = lse.view(B, hkv, L, hq // hkv).permute(0, 1, 3, 2).reshape(B, hq, L)
    s["o"].copy_(torch.where(real[..., None, None], o.to(s["o"].dtype), s["o"]))
    s["lse"].copy_(torch.where(real[:, None], lse, s["lse"]))
    return s["o"], s["lse"]


def _attn(s):
    c = s["case"]
    idx = torch.arange(s["table"].shape[1], device="cuda").expand(c["batch"], c["heads_kv"], -1)
    return _attend(s, idx)


def _sparse(s):
    c = s["case"]
    B, L, hq, d, hkv, R, P = c["batch"], c["new_len"], c["heads_q"], c["head_dim"], c["heads_kv"], c["page_rows"], s["table"].shape[1]
    # Scores in 64 bits: pages next to the border are told apart by the last bits.
    q = s["q"].double().view(B, L, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4)
    q = q.masked_fill((torch.arange(L, device="cuda")[None] >= s["new_rows"][:, None])[:, None, :, None, None], 0).flatten(2, 3)
    bounds = s["bounds"][s["table"].long()].double().permute(0, 2, 3, 4, 1)     # [B][H_kv][2][d][P]
    bounds = bounds.masked_fill(~torch.isfinite(bounds), 0)                      # pages in no table
    score = (q.clamp(min=0) @ bounds[:, :, 1] + q.clamp(max=0) @ bounds[:, :, 0])
    hidden = (torch.arange(L, device="cuda")[None] >= s["new_rows"][:, None]).repeat_interleave(hq // hkv, 1)
    score = score.masked_fill(hidden[:, None, :, None], -math.inf).amax(2)
    page = torch.arange(P, device="cuda")[None, None]
    n = ((s["kv_len"] + R - 1) // R)[:, None, None]
    score = score.masked_fill((page < c["first"]) | (page >= n - c["last"]), math.inf).masked_fill(page >= n, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :c["top_k"]]
    best = torch.sort(best.masked_fill(best >= n, P), -1)[0]
    if best.shape[-1] < c["top_k"]:
        best = torch.nn.functional.pad(best, (0, c["top_k"] - best.shape[-1]), value=P)
    s["page_idx"].copy_(best.masked_fill(best == P, -1))
    return (s["page_idx"], *_attend(s, s["page_idx"]))


# ------------------------------------------------------------------------------------------- in 64 bits

def _held(s, name, page, head):
    """The rows [R][d] of one page and head, as what they stand for, in 64 bits."""
    x = s[name][page, head].double()
    if name + "_exp" in s:
        x = x * torch.pow(2.0, s[name + "_exp"][page, head].double() - 127)[..., None]
    return x


def exact(case, seed):
    s, c = prepare(case, seed), case
    d, hq, hkv, R = c["head_dim"], c["heads_q"], c["heads_kv"], c["page_rows"]
    if c["op"] == "norm":
        out = []
        for x, w in ((s["q"], s["w_q"]), (s["k"], s["w_k"])):
            x = x.double()
            x = x / (x.pow(2).sum(-1, keepdim=True) / d + _EPS).sqrt() * w.double()
            turn = s["pos"].double()[:, None] * torch.exp(torch.arange(d // 2, device="cuda").double() * (-2 / d * math.log(_BASE)))
            z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.polar(torch.ones_like(turn), turn)[:, None]
            out.append(torch.cat([z.real, z.imag], -1))
        return tuple(out)
    lens, new = _lengths(c), _new_rows(c)
    table = s["table"].cpu()
    if c["op"] == "append":
        if c["batch"] * max(_pages(c, m) + 1 for m in new) > 20000:
            return None
        for b in range(c["batch"]):
            for j in range((lens[b] - new[b]) // R, _pages(c, lens[b])):
                first, last = max(0, lens[b] - new[b] - j * R), min(R, lens[b] - j * R)
                page, r0 = int(table[b, j]), j * R + first - (lens[b] - new[b])
                for n in ("k", "v"):
                    x = s[n + "_new"][b, r0:r0 + last - first].transpose(0, 1)
                    if c["cache"] == "fp8":
                        e = torch.ceil(torch.log2(x.double().abs().amax(-1).clamp(min=2.0 ** -140) / 448)).clamp(-100, 120)
                        s[n + "_exp"][page, :, first:last] = (e + 127).to(torch.uint8)
                        x = (x.double() * torch.pow(2.0, -e)[..., None]).float().to(torch.float8_e4m3fn)
                        s[n].view(torch.uint8)[page, :, first:last] = x.view(torch.uint8)
                    else:
                        s[n][page, :, first:last] = x
                if c["bounds"]:
                    x = s["k_new"][b, r0:r0 + last - first]
                    if first > 0:
                        x = torch.cat([s["bounds"][page].transpose(0, 1), x])
                    s["bounds"][page] = torch.stack([x.amin(0), x.amax(0)], 1)
        kept = _pool(s)
        return {n: kept[n].double() if n in ("k", "v", "bounds") else None for n in kept}
    if c["op"] == "read":
        if c["batch"] * hkv * max(_pages(c, n) for n in lens) > 4_000_000:
            return None
        out = {n: s[n + "_out"].double() for n in ("k", "v")}
        for b in range(c["batch"]):
            pages = s["table"][b, :_pages(c, lens[b])].long()
            for h in range(hkv):
                for n in ("k", "v"):
                    out[n][b, h, :lens[b]] = _held(s, n, pages, h).reshape(-1, d)[:lens[b]]
        return out["k"], out["v"]
    if c["batch"] * hkv > 4096:
        return None
    L, G = c["new_len"], hq // hkv
    o, lse = s["o"].double(), s["lse"].double()
    for b in range(c["batch"]):
        count, m = _pages(c, lens[b]), new[b]
        for h in range(hkv):
            q = s["q"][b, :m, h * G:(h + 1) * G].double()
            keep = torch.arange(count, device="cuda")
            if c["op"] == "sparse":
                lo, hi = s["bounds"][s["table"][b, :count].long(), h].double().unbind(1)
                best = torch.stack([torch.where(r >= 0, r * hi, r * lo).sum(-1) for r in q.reshape(-1, d)]).amax(0)
                best[:c["first"]] = math.inf
                best[max(0, count - c["last"]):] = math.inf
                keep = torch.sort(torch.sort(best, descending=True, stable=True)[1][:c["top_k"]])[0]
                s["page_idx"][b, h] = -1
                s["page_idx"][b, h, :len(keep)] = keep
            pages = s["table"][b, keep].long()
            at = (keep[:, None] * R + torch.arange(R, device="cuda")).reshape(-1)
            fits = at < lens[b]
            k, v = (_held(s, n, pages, h).reshape(-1, d)[fits] for n in ("k", "v"))
            end = lens[b] - m + 1 + torch.arange(m, device="cuda") if c["causal"] else torch.full((m,), lens[b], device="cuda")
            z = torch.matmul(q, k.t()) / math.sqrt(d)
            z = torch.where((at[fits] < end[:, None])[:, None], z, -math.inf)
            lse[b, h * G:(h + 1) * G, :m] = torch.logsumexp(z, -1).t()
            w = torch.softmax(z, -1)
            o[b, :m, h * G:(h + 1) * G] = torch.matmul(w, v)
    return (None, o, lse) if c["op"] == "sparse" else (o, lse)
