"""More operators of the paged key/value cache, in plain form and through the binding, and the cases that they are timed on.

* ``attn``   -- pd_paged_attn over a cache held in 4 bits;
* ``write``  -- pd_paged_append of rows into a cache of 4 bits, then pd_paged_read of all rows as what they stand for;
* ``window`` -- pd_paged_window_attn: a sliding window and a few first positions that stay visible;
* ``rope``   -- pd_paged_append_rope: the rows of a projection into the pages, with the head norms and the rotary
  positions on the way (a cache of 4 bits is read back, as in ``write``).

A cache of 4 bits holds E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two a byte with the even channel in the
low half, times a power of two for every 32 channels of a head's row, whose exponent e is kept as the byte e + 127: the
least e with max|x| <= 6 * 2^e, within -100..126.  One of 8 bits holds E4M3 values times a power of two for a head's row: the
least e with max|x| <= 448 * 2^e, within -100..120.
"""

import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}
_EPS = 1e-6
_BASE = 5e5

_DEFAULT = {"op": "attn", "dtype": "bf16", "cache": "fp4", "batch": 1, "new_len": 1, "kv_len": 8192, "ragged": False,
            "heads_q": 32, "heads_kv": 32, "head_dim": 128, "page_rows": 64, "causal": True, "bounds": True,
            "window": 0, "sinks": 0, "given": False}


def _case(name=None, **kw):
    c = dict(_DEFAULT, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # The next token of one 8K request, 7 query heads per key head: the latency of a call.
        _case("attn4_token_8k_gqa", heads_q=28, heads_kv=4),
        # A serving batch of 64 requests of 512 to 32K rows, small pages, 4 query heads per key head.
        _case("attn4_serving", batch=64, kv_len=32768, ragged=True, heads_kv=8, page_rows=16),
        # The next tokens of eight 32K requests with as many key heads as query heads: the largest call.
        _case("attn4_token_32k_b8", batch=8, kv_len=32768),
        # A few odd rows of two short prompts, d = 64, into 4 bits and back.
        _case("write4_short_d64", op="write", batch=2, new_len=37, kv_len=101, heads_q=8, heads_kv=4, head_dim=64,
              page_rows=32, bounds=False),
        # Prompts of four requests, of odd lengths up to 4161 rows, into 4 bits and back as a prefix in bf16.
        _case("write4_prompt", op="write", batch=4, new_len=4161, kv_len=4161, ragged=True),
        # The next token of one 8K request within a window of 1024: as much work at any length.
        _case("window_token_8k_gqa", op="window", cache="bf16", heads_q=28, heads_kv=4, window=1024, sinks=4),
        # A serving batch of 64 requests of up to 32K rows, 8-bit cache, window of 4096.
        _case("window_serving_fp8", op="window", cache="fp8", batch=64, kv_len=32768, ragged=True, heads_kv=8, page_rows=16,
              window=4096, sinks=4),
        # A denoising block of 32 rows that see each other, full precision, d = 64, an odd window.
        _case("window_block32_fp32", op="window", dtype="fp32", cache="fp32", batch=2, new_len=32, kv_len=1000, ragged=True,
              heads_q=8, heads_kv=4, head_dim=64, page_rows=32, causal=False, window=301, sinks=5),
        # A chunk of a prompt, 512 rows behind 7.5K others, window of 1024: matrix products count.
        _case("window_chunk512", op="window", cache="bf16", new_len=512, heads_kv=8, window=1024, sinks=16),
        # A decoding step of eight requests of different lengths, 8-bit cache.
        _case("rope_token_fp8", op="rope", cache="fp8", batch=8, ragged=True, heads_q=28, heads_kv=4),
        # The tokens of an odd batch of short prompts at positions of their own, full precision, d = 64.
        _case("rope_ragged_fp32_d64", op="rope", dtype="fp32", cache="fp32", batch=3, new_len=777, kv_len=777, ragged=True,
              heads_q=12, heads_kv=4, head_dim=64, page_rows=32, given=True),
        # Prompts of four requests, of odd lengths up to 4161 rows.
        _case("rope_prompt", op="rope", cache="bf16", batch=4, new_len=4161, kv_len=4161, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["attn", "attn", "write", "window", "window", "rope", "rope"])
        dtype = "bf16" if op in ("attn", "write") else rng.choice(["bf16", "bf16", "bf16", "fp32"])
        hkv = rng.choice([1, 2, 4, 8, 32])
        hq = hkv * (rng.choice([1, 2, 4, 7, 8]) if hkv < 32 else 1)
        cache = "fp4" if op in ("attn", "write") else "fp32" if dtype == "fp32" else rng.choice(["bf16", "fp8", "fp4"])
        case = _case(op=op, dtype=dtype, cache=cache, batch=_log(rng, 1, 64), kv_len=_log(rng, 33, 131072),
                     ragged=rng.random() < 0.6, heads_q=hq, heads_kv=hkv, head_dim=rng.choice([64, 128, 128]),
                     page_rows=rng.choice([16, 32, 64, 64, 128, 256]), causal=rng.random() < 0.7)
        if op == "attn":
            case.update(new_len=rng.choice([1, 1, 1, rng.randint(2, 33)]))
        elif op == "window":
            case.update(new_len=rng.choice([1, 1, rng.randint(2, 33), _log(rng, 33, 512)]), window=_log(rng, 1, 8192),
                        sinks=rng.choice([0, 1, 4, rng.randint(0, 64)]))
        else:
            if op == "write" or cache == "fp4":
                case["kv_len"] = min(case["kv_len"], 8192)    # all rows are read back
            case.update(new_len=rng.choice([1, _log(rng, 1, case["kv_len"])]), bounds=rng.random() < 0.7,
                        given=rng.random() < 0.3)
        w, rows = work(case), sum(_lengths(case))
        # A plain form holds every key in sight in 32 bits, and a weight for each query row and key.
        if op == "window":
            rows = case["batch"] * min(case["kv_len"], case["sinks"] + case["window"] + case["new_len"])
        if (w["bytes"] <= largest and w["flops"] <= 4e10 and rows * hkv * case["head_dim"] <= 1 << 30
                and sum(_lengths(case)) * hkv * case["head_dim"] <= 1 << 31):
            return case


# ------------------------------------------------------------------------------------------- sizes

def _lengths(c):
    """Rows of each sequence, the new ones included: spread evenly up to kv_len in a scattered order, or all kv_len."""
    B, n = c["batch"], c["kv_len"]
    if not c["ragged"]:
        return [n] * B
    least = 1 if c["op"] in ("write", "rope") else c["new_len"]   # prompts may be shorter than the places for new rows
    step = 37 if B % 37 else 1
    return [max(least, n * (b * step % B + 1) // B) for b in range(B)]


def _new_rows(c):
    return [min(c["new_len"], n) for n in _lengths(c)]


def _pages(c, n):
    return -(-n // c["page_rows"])


def _row_bytes(c):
    """One head's row in the cache."""
    d = c["head_dim"]
    return {"fp4": d // 2 + d // 32, "fp8": d + 1, "bf16": 2 * d, "fp32": 4 * d}[c["cache"]]


def work(case):
    """Bytes and operations that one pass cannot do without: inputs read once, outputs written once."""
    c = case
    eb, d, hq, hkv, row = _BYTES[c["dtype"]], c["head_dim"], c["heads_q"], c["heads_kv"], _row_bytes(c)
    lens, new = _lengths(c), _new_rows(c)
    if c["op"] in ("write", "rope"):
        n = sum(new) * hkv * 2
        touched = sum(_pages(c, s) - (s - m) // c["page_rows"] for s, m in zip(lens, new))
        by, fl = n * (d * eb + row) + (touched * hkv * 2 * d * eb if c["bounds"] else 0), 4 * n * d
        if c["op"] == "rope":
            by += sum(new) * (hq * 2 * d * eb + (4 if c["given"] else 0))
            fl += 8 * sum(new) * (hq + hkv) * d
        if c["cache"] == "fp4":
            by += sum(lens) * hkv * 2 * (d * eb + row)
        return {"bytes": by, "flops": fl}
    by = fl = 0
    for s, m in zip(lens, new):
        first = max(0, s - m - c["window"] + 1) if c["op"] == "window" else 0
        rows = min(s, s - first + min(c["sinks"], first))
        seen = 0
        for p in range(s - m, s):
            end = p + 1 if c["causal"] else s
            low = max(0, p - c["window"] + 1) if c["op"] == "window" else 0
            seen += end - low + min(c["sinks"], low)
        by += rows * hkv * 2 * row + m * hq * (2 * d * eb + 4)
        fl += 4 * seen * hq * d
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _quantised(x, kind):
    """Rows [..., d] as the bytes of the pages, and their exponent bytes: [...] in 8 bits, [..., d / 32] in 4."""
    if kind == "fp8":
        m, e = torch.frexp(x.abs().amax(-1))       # m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
        e = torch.where(m == 0, -100, e - 9 + (m > 0.875).to(e.dtype)).clamp(-100, 120)
        return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)
    x = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))           # 6 = 0.75 * 2^3
    e = torch.where(m == 0, -100, e - 3 + (m > 0.75).to(e.dtype)).clamp(-100, 126)
    x = torch.ldexp(x, -e[..., None])
    a = x.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step               # ties to even
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = (code + 8 * torch.signbit(x).to(torch.uint8)).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def prepare(case, seed):
    c, g = case, _gen(seed)
    t, d, hq, hkv, R, B = _TYPES[c["dtype"]], c["head_dim"], c["heads_q"], c["heads_kv"], c["page_rows"], c["batch"]
    s = {"case": c}
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
    k, v = k.to(t), v.to(t)
    if c["op"] in ("write", "rope") and c["bounds"]:
        # Bounds of the rows that the sequences hold.
        page_len = torch.full((used + 1,), R, device="cuda")
        page_len[order[(starts + counts - 1)].long()] = s["kv_len"].long() - (counts - 1) * R
        hidden = (torch.arange(R, device="cuda")[None] >= page_len[:, None])[:, None, :, None]
        s["bounds"] = torch.stack([k.masked_fill(hidden, math.inf).amin(2), k.masked_fill(hidden, -math.inf).amax(2)], 2).contiguous()
    if c["cache"] in ("fp8", "fp4"):
        for n, x in (("k", k), ("v", v)):
            s[n], e = _quantised(x.float(), c["cache"])
            s[n + "_exp"] = e if c["cache"] == "fp8" else e.transpose(2, 3).contiguous()   # [pages][H_kv][d / 32][R]
        if c["cache"] == "fp8":
            s["k"], s["v"] = s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn)
    else:
        s["k"], s["v"] = k, v
    del k, v
    if c["op"] in ("write", "rope"):
        # The rows of a fused projection [q | k | v], or [k | v].
        lead = hq if c["op"] == "rope" else 0
        fused = (_normal(g, B, c["new_len"], lead + 2 * hkv, d) * 1.5).to(t)
        s["q"], s["k_new"], s["v_new"] = fused[:, :, :lead], fused[:, :, lead:lead + hkv], fused[:, :, lead + hkv:]
        if c["op"] == "rope":
            s["w_q"], s["w_k"] = ((1 + 0.2 * _normal(g, d)).to(t) for _ in range(2))
            s["q_out"] = torch.zeros((B, c["new_len"], hq, d), dtype=t, device="cuda")
            s["pos"] = None
            if c["given"]:
                s["pos"] = ((torch.arange(B * c["new_len"], device="cuda") * 3 + int(seed) % 1000) % 131072).to(torch.int32).view(B, -1)
        if c["cache"] == "fp4":
            s["k_out"], s["v_out"] = (torch.zeros((B, hkv, max(lens), d), dtype=t, device="cuda") for _ in range(2))
    else:
        s["q"] = _normal(g, B, c["new_len"], hq, d).to(t)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, hq, c["new_len"]), device="cuda")
    return s


# ------------------------------------------------------------------------------------------- the passes

def run(state):
    if own:
        return _own(state)
    return {"attn": _attn, "write": _write, "window": _window, "rope": _rope}[state["case"]["op"]](state)


def _plan(s):
    """Sizes, cache descriptor and workspace, as a program keeps them."""
    from paper_2606_10537_amd import _lib
    c = s["case"]
    kinds = {"bf16": _lib.PD_BF16, "fp32": _lib.PD_FP32, "fp8": _lib.PD_FP8_E4M3, "fp4": _lib.PD_FP4_E2M1}
    dims = _lib.PagedDims(batch=c["batch"], new_len=c["new_len"], n_heads_q=c["heads_q"], n_heads_kv=c["heads_kv"],
                          head_dim=c["head_dim"], dtype=kinds[c["dtype"]], cache_dtype=kinds[c["cache"]],
                          page_rows=c["page_rows"], n_pages=s["k"].shape[0], max_pages=s["table"].shape[1],
                          causal=int(c["causal"]))
    cache = _lib.PagedCache(dims, s["k"], s["v"], s["table"], s["kv_len"], new_rows=s["new_rows"], k_exp=s.get("k_exp"),
                            v_exp=s.get("v_exp"), k_bounds=s.get("bounds"))
    n = 0
    if c["op"] == "attn":
        n = _lib.pd_paged_workspace_bytes(dims, 0, 1)
    elif c["op"] == "window":
        n = _lib.pd_paged_window_workspace_bytes(dims, c["window"], c["sinks"])
    return dims, cache, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _own(s):
    from paper_2606_10537_amd import _lib
    c = s["case"]
    if "plan" not in s:
        s["plan"] = _plan(s)
    dims, cache, ws = s["plan"]
    if c["op"] == "attn":
        _lib.pd_paged_attn(dims, cache, s["q"], s["o"], s["lse"], workspace=ws)
        return s["o"], s["lse"]
    if c["op"] == "window":
        _lib.pd_paged_window_attn(dims, cache, s["q"], c["window"], c["sinks"], s["o"], s["lse"], workspace=ws)
        return s["o"], s["lse"]
    if c["op"] == "rope":
        _lib.pd_paged_append_rope(dims, cache, s["q"], s["k_new"], s["v_new"], s["w_q"], s["w_k"], _EPS, s["pos"], _BASE,
                                  s["q_out"])
    else:
        _lib.pd_paged_append(dims, cache, s["k_new"], s["v_new"])
    if c["cache"] == "fp4":
        _lib.pd_paged_read(dims, cache, 0, s["k_out"].shape[2], s["k_out"], s["v_out"])
    return _written(s)


def _written(s):
    """What the rows that were written stand for: the pages (the spare page takes the plain form's padding rows), or in 4
    bits the rows read back."""
    names = ("k_out", "v_out") if s["case"]["cache"] == "fp4" else ("k", "v", "k_exp", "v_exp")
    out = {n: s[n] if n.endswith("out") else s[n][:-1] for n in names + ("bounds",) if n in s}
    if "q_out" in s:
        out["q_out"] = s["q_out"]
    return out


def _values(s, name, page, head, slot):
    """Rows of the pages in 32 bits, as what they stand for.  The indices are broadcast against each other."""
    x = s[name][page, head, slot]
    kind = s["case"]["cache"]
    if kind == "fp8":
        return torch.ldexp(x.float(), (s[name + "_exp"][page, head, slot].int() - 127)[..., None])
    if kind == "fp4":
        e = s[name + "_exp"].transpose(2, 3)[page, head, slot].int() - 127
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
        table = torch.cat([table, -table])
        pair = torch.stack([table.repeat(16), table.repeat_interleave(16)], -1)       # of a byte
        return torch.ldexp(pair[x.int()].flatten(-2).unflatten(-1, (-1, 32)), e[..., None]).flatten(-2)
    return x.float()


def _attend(s, pos):
    """Attention over the positions pos [B][n] (-1: none), each at most once, that a row sees."""
    c = s["case"]
    B, L, hq, d, hkv, R = c["batch"], c["new_len"], c["heads_q"], c["head_dim"], c["heads_kv"], c["page_rows"]
    at = pos.clamp(min=0)
    page = s["table"].gather(1, at // R).long()[:, None]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    k, v = (_values(s, n, page, head, (at % R)[:, None]) for n in ("k", "v"))
    q = s["q"].float().view(B, L, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [B][H_kv][L * G][d]
    row = torch.arange(L, device="cuda")[None]
    own_pos = s["kv_len"][:, None] - s["new_rows"][:, None] + row
    end = own_pos + 1 if c["causal"] else s["kv_len"][:, None] + 0 * row
    seen = (pos >= 0)[:, None] & (pos[:, None] < end[..., None])
    if c["op"] == "window":
        seen &= (pos < c["sinks"])[:, None] | (pos[:, None] > own_pos[..., None] - c["window"])
    seen = seen.repeat_interleave(hq // hkv, 1)[:, None]
    w = ((q @ k.transpose(2, 3)) * d ** -0.5).masked_fill_(~seen, -math.inf)
    del k
    top = w.amax(-1, keepdim=True).clamp(min=-1e30)
    w = torch.exp_(w.sub_(top))
    total = w.sum(-1, keepdim=True)
    v.masked_fill_(~((pos >= 0) & (pos < s["kv_len"][:, None]))[:, None, :, None], 0)
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
    pos = torch.arange(c["kv_len"], device="cuda").expand(c["batch"], -1)
    return _attend(s, torch.where(pos < s["kv_len"][:, None], pos, -1))


def _window(s):
    # The first positions, where they lie before the window of the first new row, and the windows of all new rows.
    c = s["case"]
    low = (s["kv_len"] - s["new_rows"] - c["window"] + 1).clamp(min=0)[:, None]
    first = torch.arange(min(c["sinks"], c["kv_len"]), device="cuda")[None]
    near = low + torch.arange(min(c["window"] + c["new_len"] - 1, c["kv_len"]), device="cuda")[None]
    return _attend(s, torch.cat([torch.where(first < low, first, -1), torch.where(near < s["kv_len"][:, None], near, -1)], 1))


def _put(s, k, v):
    """Rows k, v [B][L][H_kv][d] (dtype) into the pages, with the bounds of the keys."""
    c = s["case"]
    R, spare = c["page_rows"], s["k"].shape[0] - 1
    r = torch.arange(c["new_len"], device="cuda")
    real = r[None] < s["new_rows"][:, None]
    pos = (s["kv_len"] - s["new_rows"])[:, None] + r[None]
    page = torch.where(real, s["table"].gather(1, (pos // R).clamp(0, s["table"].shape[1] - 1).long()), spare).long().reshape(-1)
    slot = torch.where(real, pos % R, 0).long().reshape(-1)
    for name, x in (("k", k.flatten(0, 1)), ("v", v.flatten(0, 1))):
        if c["cache"] in ("fp8", "fp4"):
            x, e = _quantised(x.float(), c["cache"])
            s[name].view(torch.uint8)[page, :, slot] = x
            if c["cache"] == "fp8":
                s[name + "_exp"][page, :, slot] = e
            else:
                s[name + "_exp"][page, :, :, slot] = e
        else:
            s[name][page, :, slot] = x
    if c["bounds"]:
        x, old = k.flatten(0, 1).float(), s["bounds"].float()
        low = torch.full_like(old[:, :, 0], math.inf).index_reduce_(0, page, x, "amin")
        high = torch.full_like(old[:, :, 1], -math.inf).index_reduce_(0, page, x, "amax")
        fresh = torch.zeros(spare + 1, device="cuda").index_put_((page,), (slot == 0).float(), accumulate=True) > 0
        fresh = fresh[:, None, None]   # a page whose first row is written begins anew
        low = torch.where(fresh, low, torch.minimum(old[:, :, 0], low))
        high = torch.where(fresh, high, torch.maximum(old[:, :, 1], high))
        s["bounds"].copy_(torch.stack([low, high], 2))


def _back(s):
    """All rows of a cache of 4 bits into k_out, v_out."""
    c = s["case"]
    n, R = s["k_out"].shape[2], c["page_rows"]
    pos = torch.arange(n, device="cuda")
    page = s["table"][:, pos // R].long()[:, None]
    head = torch.arange(c["heads_kv"], device="cuda")[None, :, None]
    valid = (pos[None] < s["kv_len"][:, None])[:, None, :, None]
    for name in ("k", "v"):
        out = s[name + "_out"]
        out.copy_(torch.where(valid, _values(s, name, page, head, pos % R).to(out.dtype), out))


def _write(s):
    _put(s, s["k_new"], s["v_new"])
    _back(s)
    return _written(s)


def _rope(s):
    # In 64 bits: rows next to a border of the cache's few bits, and angles of far positions.
    c = s["case"]
    t, half = _TYPES[c["dtype"]], c["head_dim"] // 2
    r = torch.arange(c["new_len"], device="cuda")[None]
    pos = (s["kv_len"] - s["new_rows"])[:, None] + r if s["pos"] is None else s["pos"]
    angle = pos.double()[:, :, None, None] * _BASE ** (torch.arange(half, device="cuda", dtype=torch.float64) / -half)
    cos, sin = torch.cos(angle), torch.sin(angle)

    def turned(x, w):
        y = x.double()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + _EPS) * w.double()
        a, b = y.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).float().to(t)

    real = (r < s["new_rows"][:, None])[..., None, None]
    s["q_out"].copy_(torch.where(real, turned(s["q"], s["w_q"]), s["q_out"]))
    _put(s, turned(s["k_new"], s["w_k"]), s["v_new"])
    if c["cache"] == "fp4":
        _back(s)
    return _written(s)


# ------------------------------------------------------------------------------------------- in 64 bits

def _nearest4(x):
    """Values within +-6 to the nearest E2M1 value, by the borders between neighbours; a border goes to the even code."""
    a, out = x.abs(), torch.zeros_like(x)
    for border, up, below in ((0.25, 0.5, True), (0.75, 1.0, False), (1.25, 1.5, True), (1.75, 2.0, False), (2.5, 3.0, True),
                              (3.5, 4.0, False), (5.0, 6.0, True)):
        out = torch.where((a > border) if below else (a >= border), up, out)
    return torch.where(x < 0, -out, out)


def _held(x, kind):
    """Rows in 64 bits as a cache of this kind holds them, and their exponents."""
    if kind == "fp8":
        e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -140) / 448)).clamp(-100, 120)
        y = x * torch.pow(2.0, -e)
        return y.float().to(torch.float8_e4m3fn).double(), e[..., 0]
    if kind == "fp4":
        g = x.reshape(*x.shape[:-1], -1, 32)
        e = torch.ceil(torch.log2(g.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -140) / 6)).clamp(-100, 126)
        return (_nearest4(g * torch.pow(2.0, -e)) * torch.pow(2.0, e)).reshape(x.shape), e[..., 0]
    return x, None


def _stored(s, name, b, h, n):
    """Rows 0..n-1 of sequence b and KV head h, as what they stand for, in 64 bits."""
    c = s["case"]
    pages = s["table"][b, :_pages(c, n)].long()
    x = s[name][pages, h]
    if c["cache"] == "fp4":
        codes = torch.stack([x & 15, x >> 4], -1).flatten(-2).long()
        x = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")[codes % 8] * (1 - 2 * (codes // 8))
        e = s[name + "_exp"][pages, h].double() - 127
        x = x * torch.pow(2.0, e).transpose(1, 2).repeat_interleave(32, -1)
    else:
        x = x.double()
        if c["cache"] == "fp8":
            x = x * torch.pow(2.0, s[name + "_exp"][pages, h].double() - 127)[..., None]
    return x.reshape(-1, x.shape[-1])[:n]


def _exact_written(s):
    c = s["case"]
    d, hq, R, t = c["head_dim"], c["heads_q"], c["page_rows"], _TYPES[c["dtype"]]
    lens, new = _lengths(c), _new_rows(c)
    if c["batch"] * max(_pages(c, m) + 1 for m in new) > 20000:
        return None
    quant = c["cache"] in ("fp8", "fp4")
    out = {n: x.double() for n, x in _written(s).items()}
    rows = {}
    for b in range(c["batch"]):
        m, start = new[b], lens[b] - new[b]
        q, k, v = (s[n][b, :m].double() for n in ("q", "k_new", "v_new"))
        if c["op"] == "rope":
            where = s["pos"][b, :m].double() if c["given"] else start + torch.arange(m, device="cuda", dtype=torch.float64)
            turn = where[:, None] * torch.exp(torch.arange(d // 2, device="cuda").double() * (-2 / d * math.log(_BASE)))
            for x, w in ((q, s["w_q"]), (k, s["w_k"])):
                x /= (x.pow(2).sum(-1, keepdim=True) / d + _EPS).sqrt()
                x *= w.double()
                z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * torch.polar(torch.ones_like(turn), turn)[:, None]
                x.copy_(torch.cat([z.real, z.imag], -1))
            out["q_out"][b, :m] = q
        # Keys are rounded to the type of the rows before they are held in fewer bits.
        held = k.float().to(t).double() if quant else k
        rows[b] = {"k": _held(held, c["cache"]), "v": _held(v, c["cache"])}
        for j in range(start // R, _pages(c, lens[b])):
            first, last = max(0, start - j * R), min(R, lens[b] - j * R)
            page, r0 = int(s["table"][b, j]), j * R + first - start
            if c["bounds"]:
                x = held[r0:r0 + last - first]
                if first > 0:
                    x = torch.cat([out["bounds"][page].transpose(0, 1), x])
                out["bounds"][page] = torch.stack([x.amin(0), x.amax(0)], 1)
            if c["cache"] != "fp4":
                for n in ("k", "v"):
                    out[n][page, :, first:last] = rows[b][n][0][r0:r0 + last - first].transpose(0, 1)
    if c["cache"] == "fp4":
        for b in range(c["batch"]):
            for n in ("k", "v"):
                for h in range(c["heads_kv"]):
                    out[n + "_out"][b, h, :lens[b]] = _stored(s, n, b, h, lens[b])
                out[n + "_out"][b, :, lens[b] - new[b]:lens[b]] = rows[b][n][0].transpose(0, 1)
    for n in ("k_exp", "v_exp"):
        if n in out:
            out[n] = None
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] in ("write", "rope"):
        return _exact_written(s)
    d, hq, hkv = c["head_dim"], c["heads_q"], c["heads_kv"]
    lens, new = _lengths(c), _new_rows(c)
    if c["batch"] * hkv > 4096:
        return None
    G = hq // hkv
    o, lse = s["o"].double(), s["lse"].double()
    for b in range(c["batch"]):
        n, m = lens[b], new[b]
        at, row = torch.arange(n, device="cuda")[None], torch.arange(n - m, n, device="cuda").repeat_interleave(G)[:, None]
        fits = (at <= row) if c["causal"] else (at < n)
        if c["op"] == "window":
            fits = fits & ((row - at < c["window"]) | (at < c["sinks"]))
        for h in range(hkv):
            q = s["q"][b, :m, h * G:(h + 1) * G].double().reshape(-1, d)
            k, v = (_stored(s, x, b, h, n) for x in ("k", "v"))
            z = torch.matmul(q, k.t()) / math.sqrt(d)
            z = torch.where(fits, z, -math.inf)
            lse[b, h * G:(h + 1) * G, :m] = torch.logsumexp(z, -1).view(m, G).t()
            o[b, :m, h * G:(h + 1) * G] = torch.matmul(torch.softmax(z, -1), v).view(m, G, d)
    return o, lse
