"""The operators of the paged key/value cache, as timed cases.

A program that feeds a language model in chunks (images first, text as it
arrives, then token by token) keeps every request's keys and values in pages of
one pool.  Per layer and chunk it normalises and rotates the queries and keys
(``qk_norm_rope``), appends the new keys and values to the pages
(``paged_append``) and lets the new tokens attend to everything the request has
in the cache (``paged_attention``); an action expert then reads the cache as
one contiguous prefix per request (``paged_gather``).

Batches are padded: request b has ``new_len[b]`` valid rows of ``rows``; rows
behind them are left as they were.  Lengths are part of a case, so that its work
is known; values, page order and weights are made from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
ROPE_BASE = 10000.0
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "fp8": 1}
FP8_MAX = 448.0


def attention(name, batch, rows, heads, kv_heads, dim, page, kv_min, kv_max, new_min=None, dtype="bf16", kv=None,
              causal=True, window=0):
    c = {"name": name, "op": "attention", "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads,
         "dim": dim, "page": page, "kv_min": kv_min, "kv_max": kv_max, "new_min": rows if new_min is None else new_min,
         "dtype": dtype, "kv": kv or dtype, "causal": causal, "window": window}
    return c


def append(name, batch, rows, kv_heads, dim, page, past_max, new_min=None, dtype="bf16", kv=None):
    return {"name": name, "op": "append", "batch": batch, "rows": rows, "kv_heads": kv_heads, "dim": dim, "page": page,
            "past_max": past_max, "new_min": rows if new_min is None else new_min, "dtype": dtype, "kv": kv or dtype}


def norm_rope(name, batch, rows, heads, kv_heads, dim, past_max, new_min=None, dtype="bf16"):
    return {"name": name, "op": "norm_rope", "batch": batch, "rows": rows, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "past_max": past_max, "new_min": rows if new_min is None else new_min, "dtype": dtype}


def gather(name, layers, batch, rows, kv_heads, dim, page, len_min, kv="bf16"):
    return {"name": name, "op": "gather", "layers": layers, "batch": batch, "rows": rows, "kv_heads": kv_heads,
            "dim": dim, "page": page, "len_min": len_min, "kv": kv}


def listed():
    return [
        # one request, one new token over the 816-token prefix of a policy with one K/V head: latency alone
        attention("attend_token_b1", 1, 1, 8, 1, 256, 64, 817, 817),
        # a serving batch of single tokens over ragged contexts, small pages
        attention("attend_tokens_b64", 64, 1, 32, 8, 128, 16, 600, 4000),
        # few requests, very long contexts, the cache held in 8 bits
        attention("attend_long_fp8_b4", 4, 1, 32, 8, 128, 64, 90001, 131072, kv="fp8"),
        # a long prompt fed in chunks: the second chunk of 4,096 tokens (the largest)
        attention("attend_chunk_4096", 1, 4096, 32, 8, 128, 64, 8192, 8192),
        # the observation prefix as one chunk, every token seeing every token, ragged
        attention("attend_prefix_b4", 4, 816, 8, 1, 256, 64, 600, 816, new_min=600, causal=False),
        # the 32-bit path: short ragged chunks behind a sliding window
        attention("attend_window_f32_b3", 3, 37, 4, 2, 64, 16, 150, 301, new_min=11, dtype="f32", window=96),
        # a prompt chunk of eight requests into the pages, keys rotated on the way
        append("append_chunk_b8", 8, 2048, 8, 128, 64, 4097, new_min=1500),
        # single tokens of a serving batch into an 8-bit cache
        append("append_tokens_fp8_b64", 64, 1, 8, 128, 16, 4000, kv="fp8"),
        # queries and keys of two long chunks far into a context
        norm_rope("norm_rope_chunk_b2", 2, 4096, 32, 8, 128, 100000, new_min=3500),
        # queries and keys of a few tokens on the 32-bit path
        norm_rope("norm_rope_f32_b5", 5, 3, 4, 1, 64, 517, dtype="f32"),
        # the 18-layer prefix of eight requests for the action expert
        gather("gather_prefix_b8", 18, 8, 816, 1, 256, 64, 600),
        # the same for one request from an 8-bit cache, two K/V heads
        gather("gather_prefix_fp8_b1", 18, 1, 816, 2, 128, 16, 761, kv="fp8"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "norm_rope", "gather"])
    dim = rng.choice([64, 128, 256])
    kv_heads = rng.choice([1, 1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128, 256])
    dtype, kv = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
    if op == "attention":
        causal = rng.random() < 0.8
        window = _log(rng, 16, 4096) if causal and rng.random() < 0.25 else 0
        if rng.random() < 0.5:                       # a few new tokens, many keys
            rows = _log(rng, 1, 8)
            batch = _log(rng, 1, 64)
            # at most 2^29 bytes of keys and values
            most = (1 << 29) // (batch * kv_heads * dim * 2 * BYTES[kv])
        else:                                        # a chunk
            rows = _log(rng, 9, 4096)
            batch = _log(rng, 1, max(1, min(64, 16384 // rows)))
            # at most 2^29 pairs of a query head's row and a key (32 bits: a quarter of that)
            most = (1 << (27 if dtype == "f32" else 29)) // (batch * rows * group * kv_heads)
        most = max(rows, min(65536, most))
        kv_max = _log(rng, rows, most) if most > rows else rows
        kv_min = max(1, int(kv_max * rng.uniform(0.3, 1.0)))
        new_min = max(1, int(rows * rng.uniform(0.3, 1.0)))
        c = attention("", batch, rows, group * kv_heads, kv_heads, dim, page, kv_min, kv_max, new_min, dtype, kv,
                      causal, window)
    elif op == "append":
        rows = _log(rng, 1, 2048)
        batch = _log(rng, 1, max(1, min(64, 16384 // rows)))
        c = append("", batch, rows, kv_heads, dim, page, _log(rng, 1, 8192), max(1, int(rows * rng.uniform(0.3, 1.0))),
                   dtype, kv)
    elif op == "norm_rope":
        rows = _log(rng, 1, 4096)
        batch = _log(rng, 1, max(1, min(64, 8192 // rows)))
        c = norm_rope("", batch, rows, group * kv_heads, kv_heads, dim, _log(rng, 1, 1 << 20),
                      max(1, int(rows * rng.uniform(0.3, 1.0))), dtype)
    else:
        rows = _log(rng, 16, 2000)
        c = gather("", rng.randint(1, 24), _log(rng, 1, 8), rows, kv_heads, dim, page,
                   max(1, int(rows * rng.uniform(0.3, 1.0))), kv)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# lengths and work, from the case alone
# ---------------------------------------------------------------------------
def _spread(lo, hi, n, start):
    """n whole numbers over lo .. hi, the first of them hi where start is 0."""
    return [hi - int((hi - lo + 0.999) * (((b + start) * 0.6180339887498949) % 1.0)) for b in range(n)]


def _lengths(c):
    """(new, past or kv): host lists of length batch."""
    new = _spread(c["new_min"], c["rows"], c["batch"], 0)
    if c["op"] == "attention":
        return new, _spread(c["kv_min"], c["kv_max"], c["batch"], 0)
    return new, _spread(0, c["past_max"], c["batch"], 0)


def _visible(c, new, kv):
    """(query, key) pairs of one request, and the keys that any of its queries sees."""
    if not c["causal"]:
        return new * kv, kv
    ends = [max(0, kv - new + i + 1) for i in range(new)]
    starts = [max(0, e - c["window"]) if c["window"] else 0 for e in ends]
    return sum(ends) - sum(starts), kv - min([kv] + [a for a, e in zip(starts, ends) if e > a])


def work(case):
    c = case
    if c["op"] == "gather":
        n = c["kv_heads"] * c["dim"]
        out = 4 if c["kv"] == "f32" else 2
        lens = sum(_spread(c["len_min"], c["rows"], c["batch"], 0))
        return {"bytes": 2 * c["layers"] * n * (lens * BYTES[c["kv"]] + c["batch"] * c["rows"] * out), "flops": 0}
    new, other = _lengths(c)
    e, D = BYTES[c["dtype"]], c["dim"]
    if c["op"] == "norm_rope":
        n = sum(new) * (c["heads"] + c["kv_heads"]) * D
        return {"bytes": 2 * n * e, "flops": 8 * n}
    if c["op"] == "append":
        n = 2 * sum(new) * c["kv_heads"] * D
        return {"bytes": n * (e + BYTES[c["kv"]]), "flops": 3 * n / 2}
    seen = [_visible(c, a, b) for a, b in zip(new, other)]
    return {"bytes": 2 * sum(new) * c["heads"] * D * e + 2 * sum(s[1] for s in seen) * c["kv_heads"] * D * BYTES[c["kv"]],
            "flops": 4 * D * c["heads"] * sum(s[0] for s in seen)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _values(g, shape, dtype, scale=1.0, offset=0.0):
    """Normal values; with `offset`, a mean of its own for each channel, as values have."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale
    if offset:
        x += offset * torch.randn(shape[-2:], generator=g, device="cuda", dtype=torch.float32)
    return x.to(TORCH[dtype])


def _pool(g, c, tokens, layers=None):
    """Pages for `tokens[b]` tokens of each request in random order, a tenth more than that, and their table;
    the entries behind a request's pages are -1."""
    need = [-(-t // c["page"]) for t in tokens]
    n_pages = sum(need) + max(1, sum(need) // 10)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = torch.tensor([0] + need[:-1], device="cuda").cumsum(0)
    at = torch.arange(max(max(need), 1), device="cuda")
    used = at[None, :] < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(used, order[(first[:, None] + at[None, :]).clamp(max=n_pages - 1)], -1).contiguous()
    shape = (n_pages, c["page"], c["kv_heads"], c["dim"])
    if layers:
        shape = (layers,) + shape
    s = {"table": table, "k_scale": None, "v_scale": None}
    if c["kv"] == "fp8":
        s["k_scale"] = 0.02 + 0.02 * torch.rand(c["kv_heads"], generator=g, device="cuda")
        s["v_scale"] = 0.02 + 0.02 * torch.rand(c["kv_heads"], generator=g, device="cuda")
        s["k"] = (_values(g, shape, "f32") / s["k_scale"][:, None]).to(TORCH["fp8"])
        s["v"] = (_values(g, shape, "f32", 1.0, 0.5) / s["v_scale"][:, None]).to(TORCH["fp8"])
    else:
        s["k"], s["v"] = _values(g, shape, c["kv"]), _values(g, shape, c["kv"], 1.0, 0.5)
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(c)}
    if c["op"] == "gather":
        lens = _spread(c["len_min"], c["rows"], c["batch"], 0)
        s |= _pool(g, c, lens, c["layers"])
        s["kv_len"] = _ints(lens)
        s["out"] = torch.empty((c["layers"], 2, c["batch"], c["rows"], c["kv_heads"] * c["dim"]), device="cuda",
                               dtype=torch.float32 if c["kv"] == "f32" else torch.bfloat16)
        return s
    new, other = _lengths(c)
    s["new_len"] = _ints(new)
    B, M, D = c["batch"], c["rows"], c["dim"]
    if c["op"] == "attention":
        s |= _pool(g, c, other)
        s["kv_len"] = _ints(other)
        # queries somewhat longer than a unit normal: rows that weigh some keys well above others
        s["q"] = _values(g, (B, M, c["heads"], D), c["dtype"], 1.5)
        s["out"] = torch.zeros_like(s["q"])
        return s
    s["past_len"] = _ints(other)
    # the projections leave q, k and v side by side in one row of each token
    if c["op"] == "append":
        s |= _pool(g, c, [a + b for a, b in zip(new, other)])
        row = _values(g, (B, M, 2 * c["kv_heads"], D), c["dtype"], 1.0, 0.3)
        s["k_new"], s["v_new"] = row[:, :, :c["kv_heads"]], row[:, :, c["kv_heads"]:]
        return s
    row = _values(g, (B, M, c["heads"] + c["kv_heads"], D), c["dtype"], 2.0, 0.3)
    s["q"], s["k"] = row[:, :, :c["heads"]], row[:, :, c["heads"]:]
    s["q_gain"] = 0.1 * torch.randn(D, generator=g, device="cuda")
    s["k_gain"] = 0.1 * torch.randn(D, generator=g, device="cuda")
    s["q_out"] = torch.zeros((B, M, c["heads"], D), device="cuda", dtype=TORCH[c["dtype"]])
    s["k_out"] = torch.zeros((B, M, c["kv_heads"], D), device="cuda", dtype=TORCH[c["dtype"]])
    return s


# ---------------------------------------------------------------------------
# the plain forms: 32 bits (angles in 64), rounded once
# ---------------------------------------------------------------------------
def _rotate(x, pos, dim):
    """x [B][M][heads][dim] float32, pos [B][M]: halves (i, i + dim/2) rotated by pos * base^(-2i/dim)."""
    i = torch.arange(dim // 2, device=x.device, dtype=torch.float64)
    angle = pos.double()[..., None] * ROPE_BASE ** (-2.0 * i / dim)
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _positions(s, rows):
    """Each row's position, and whether the row is valid."""
    i = torch.arange(rows, device="cuda")
    return s["past_len"].long()[:, None] + i[None, :], i[None, :] < s["new_len"][:, None]


def _codes(x):
    return x.view(torch.uint8) if x.dtype == TORCH["fp8"] else x


def _pages(pool, scale, table):
    """Every request's pages side by side, in 32 bits: [B][tokens][kv_heads][dim]."""
    x = _codes(pool)[table.long().clamp(min=0)]
    x = x.view(pool.dtype).float().flatten(1, 2)
    return x if scale is None else x * scale[:, None]


def _plain_attention(c, s):
    B, M, nkv, D = c["batch"], c["rows"], c["kv_heads"], c["dim"]
    G = c["heads"] // nkv
    k = _pages(s["k"], s["k_scale"], s["table"])
    key = torch.arange(k.shape[1], device="cuda")
    q = s["q"].float().view(B, M, nkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, nkv, M * G, D)
    x = (q @ k.permute(0, 2, 3, 1).contiguous()).view(B, nkv, M, G, -1)
    del k, q
    i = torch.arange(M, device="cuda")
    pos = (s["kv_len"] - s["new_len"])[:, None] + i[None, :]
    seen = (key[None, None, :] < s["kv_len"][:, None, None]) & (i[None, :] < s["new_len"][:, None])[:, :, None]
    if c["causal"]:
        seen = seen & (key[None, None, :] <= pos[:, :, None])
        if c["window"]:
            seen = seen & (key[None, None, :] > pos[:, :, None] - c["window"])
    seen = seen[:, None, :, None, :]
    x.mul_(D ** -0.5).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = _pages(s["v"], s["v_scale"], s["table"]).permute(0, 2, 1, 3).contiguous()
    o = (x.view(B, nkv, M * G, -1) @ v).view(B, nkv, M, G, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, M, nkv * G, D).to(s["out"].dtype)
    s["out"].copy_(torch.where((i[None, :] < s["new_len"][:, None])[:, :, None, None], o, s["out"]))
    return s["out"]


def _stored(x, scale, dtype):
    if dtype != TORCH["fp8"]:
        return x.to(dtype)
    return (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX).to(dtype)


def _plain_append(c, s):
    pos, valid = _positions(s, c["rows"])
    page = s["table"].long().gather(1, (pos // c["page"]).clamp(max=s["table"].shape[1] - 1))[valid]
    at = (pos % c["page"])[valid]
    k = _rotate(s["k_new"].float(), pos, c["dim"])[valid]
    _codes(s["k"])[page, at] = _codes(_stored(k, s["k_scale"], s["k"].dtype))
    _codes(s["v"])[page, at] = _codes(_stored(s["v_new"].float()[valid], s["v_scale"], s["v"].dtype))
    return {"k": s["k"], "v": s["v"]}


def _plain_norm_rope(c, s):
    pos, valid = _positions(s, c["rows"])

    def one(x, gain, out):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * (1.0 + gain)
        y = _rotate(y, pos, c["dim"]).to(out.dtype)
        out.copy_(torch.where(valid[:, :, None, None], y, out))
        return out

    return {"q": one(s["q"], s["q_gain"], s["q_out"]), "k": one(s["k"], s["k_gain"], s["k_out"])}


def _plain_gather(c, s):
    n = c["rows"]
    at = torch.arange(n, device="cuda")
    valid = (at[None, :] < s["kv_len"][:, None])[:, :, None, None]
    page = s["table"].long()[:, at // c["page"]].clamp(min=0)

    def one(pool, scale):
        x = _codes(pool)[:, page, (at % c["page"])[None, :]].view(pool.dtype).float()
        if scale is not None:
            x = x * scale[:, None]
        return torch.where(valid, x, 0.0).flatten(3)

    s["out"].copy_(torch.stack([one(s["k"], s["k_scale"]), one(s["v"], s["v_scale"])], 1))
    return s["out"]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _own(c, s):
    import paper_2608_03682_amd as px

    if c["op"] == "norm_rope":
        q, k = px.qk_norm_rope(s["q"], s["k"], s["q_gain"], s["k_gain"], eps=EPS, rope_base=ROPE_BASE,
                               past_len=s["past_len"], new_len=s["new_len"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": q, "k": k}
    if "cache" not in s:                             # a program makes its cache once
        s["cache"] = px.PagedCache(s["k"], s["v"], s["table"], s["k_scale"], s["v_scale"])
    if c["op"] == "attention":
        return px.paged_attention(s["q"], s["cache"], s["kv_len"], new_len=s["new_len"], max_kv_len=c["kv_max"],
                                  causal=c["causal"], window=c["window"], out=s["out"])
    if c["op"] == "append":
        px.paged_append(s["cache"], s["k_new"], s["v_new"], s["past_len"], new_len=s["new_len"], rope_base=ROPE_BASE)
        return {"k": s["k"], "v": s["v"]}
    return px.paged_gather(s["cache"], s["kv_len"], c["rows"], out=s["out"])


def run(state):
    c = state["case"]
    if own:
        return _own(c, state)
    return {"attention": _plain_attention, "append": _plain_append, "norm_rope": _plain_norm_rope,
            "gather": _plain_gather}[c["op"]](c, state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits, request by request
# ---------------------------------------------------------------------------
def _turn64(x, pos):
    """x [n][heads][dim] float64 as complex numbers x_i + j x_(i + dim/2), times e^(j pos w_i)."""
    half = x.shape[-1] // 2
    w = torch.exp(-math.log(ROPE_BASE) * torch.arange(half, device=x.device, dtype=torch.float64) / half)
    turn = torch.polar(torch.ones((), device=x.device, dtype=torch.float64), pos.double()[:, None] * w[None, :])
    z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * turn[:, None]
    return torch.cat([z.real, z.imag], -1)


def _decoded(pool, scale, pages, n):
    """The first n tokens of a request's pages: [n][kv_heads][dim] float64."""
    x = _codes(pool)[pages.long()].view(pool.dtype).double().reshape(-1, *pool.shape[-2:])[:n]
    return x if scale is None else x * scale.double()[:, None]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    page = c["page"] if "page" in c else 1
    if c["op"] == "gather":
        out = torch.zeros(s["out"].shape, device="cuda", dtype=torch.float64)
        for b, n in enumerate(s["kv_len"].tolist()):
            pages = s["table"][b, :-(-n // page)]
            for l in range(c["layers"]):
                out[l, 0, b, :n] = _decoded(s["k"][l], s["k_scale"], pages, n).flatten(1)
                out[l, 1, b, :n] = _decoded(s["v"][l], s["v_scale"], pages, n).flatten(1)
        return out
    new = s["new_len"].tolist()
    if c["op"] == "attention":
        D, G = c["dim"], c["heads"] // c["kv_heads"]
        out = torch.zeros(s["q"].shape, device="cuda", dtype=torch.float64)
        for b, n in enumerate(s["kv_len"].tolist()):
            pages, m = s["table"][b, :-(-n // page)], new[b]
            keys = _decoded(s["k"], s["k_scale"], pages, n)
            vals = _decoded(s["v"], s["v_scale"], pages, n)
            first = n - m + torch.arange(m, device="cuda")[:, None]
            behind = first - torch.arange(n, device="cuda")[None, :]        # how far each key lies behind the row
            hidden = torch.zeros_like(behind, dtype=torch.bool)
            if c["causal"]:
                hidden = behind < 0
                if c["window"]:
                    hidden |= behind >= c["window"]
            for h in range(c["heads"]):
                x = s["q"][b, :m, h].double() @ keys[:, h // G].t().contiguous() / math.sqrt(D)
                p = torch.softmax(x.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
                out[b, :m, h] = p @ vals[:, h // G]
        return out
    past = s["past_len"].tolist()
    if c["op"] == "norm_rope":
        got = {}
        for name, gain in (("q", s["q_gain"]), ("k", s["k_gain"])):
            got[name] = torch.zeros(s[name + "_out"].shape, device="cuda", dtype=torch.float64)
            for b, m in enumerate(new):
                x = s[name][b, :m].double()
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * (1 + gain.double())
                got[name][b, :m] = _turn64(x, past[b] + torch.arange(m, device="cuda"))
        return got
    pools = {"k": s["k"].double(), "v": s["v"].double()}
    for b, m in enumerate(new):
        pos = past[b] + torch.arange(m, device="cuda")
        where = s["table"][b].long()[pos // page], pos % page
        k, v = _turn64(s["k_new"][b, :m].double(), pos), s["v_new"][b, :m].double()
        if c["kv"] == "fp8":
            k = (k / s["k_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            v = (v / s["v_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        pools["k"][where], pools["v"][where] = k, v
    return pools
