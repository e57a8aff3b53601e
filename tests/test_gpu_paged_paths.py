"""Attention over the paged cache by its paths, on the GPU against the float64 oracle: few
rows (one wave a block), chunks and chunks of head_dim 256, each with the keys of a block in one
piece and in several.  Every test states the plan that it means, and asserts it by the workspace
that the plan asks for.  Bars as in test_gpu_paged.py."""
import numpy as np
import pytest

import oracle.paged as op
from test_gpu_paged import Cache, attention_bar, check, host, ints, px

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def shared_cache(seed, kind, nkv, D, ps, kv, B):
    """One prefix in random pages (the first of the pool is not among them), read by B requests;
    each row of the table is its own."""
    c = Cache(seed, kind, nkv, D, ps, [kv], stale=False)
    if 0 in c.host_table[0, :-(-kv // ps)]:
        free = next(p for p in range(c.n_pages) if p not in c.host_table[0])
        at = int(np.flatnonzero(c.host_table[0] == 0)[0])
        bits = lambda t: t.view(torch.uint8) if kind == "fp8" else t  # noqa: E731
        bits(c.k)[free], bits(c.v)[free] = bits(c.k)[0].clone(), bits(c.v)[0].clone()
        c.host_table[0, at] = free
    c.host_table = np.repeat(c.host_table, B, 0)
    c.table = torch.from_numpy(c.host_table).cuda()
    c.px = px().PagedCache(c.k, c.v, c.table, c.dks, c.dvs)
    return c


def queries(c, B, rows, H, seed=5):
    q = 1.5 * torch.randn(B, rows, H, c.D, generator=torch.Generator().manual_seed(seed))
    return q.to(torch.float32 if c.kind == "f32" else torch.bfloat16).cuda()


# (kind, head_dim, requests, rows, K/V heads, heads of each, keys, window, page size): a few rows (one wave a
# block), chunks, and chunks of head_dim 256; each with the keys of a block in one piece and in several.
# The first key of a block, rounded down to its tile, lies in a page before the first one that a row sees.
WINDOWS = [
    ("bf16", 64, 1, 1, 1, 2, 64, 16, 16), ("fp8", 128, 2, 1, 2, 4, 64, 16, 16), ("f32", 128, 1, 1, 1, 2, 64, 16, 16),
    ("f32", 256, 1, 1, 1, 2, 64, 16, 16),
    ("bf16", 64, 1, 3, 1, 2, 2500, 1000, 16), ("fp8", 256, 1, 3, 1, 2, 2500, 1000, 16), ("f32", 64, 1, 3, 1, 2, 2500, 1000, 16),
    ("bf16", 64, 1, 50, 1, 2, 150, 20, 16), ("bf16", 128, 2, 50, 1, 2, 150, 40, 32), ("fp8", 64, 1, 50, 1, 2, 150, 20, 16),
    ("f32", 64, 1, 34, 1, 2, 64, 4, 16),
    ("bf16", 64, 1, 50, 1, 2, 2500, 990, 16), ("fp8", 128, 1, 50, 1, 2, 2500, 990, 16), ("f32", 64, 1, 50, 1, 2, 2500, 990, 16),
    ("bf16", 256, 25, 9, 8, 1, 300, 70, 16), ("bf16", 256, 64, 9, 8, 1, 300, 70, 16), ("bf16", 256, 2, 150, 1, 2, 2500, 890, 16),
    ("fp8", 256, 1, 50, 1, 2, 150, 20, 16), ("fp8", 256, 1, 50, 1, 2, 2500, 990, 16)]


@pytest.mark.parametrize("kind,D,B,rows,nkv,G,kv,window,ps", WINDOWS)
def test_pages_before_the_window_may_be_given_back(kind, D, B, rows, nkv, G, kv, window, ps):
    """A page that no row sees any longer may have lost its number in the table: results are bit
    for bit those of the whole table, and no status bit is raised.  The first page that a row sees
    is judged."""
    kvs = [kv - 5 * (b % 3) for b in range(B)]
    c = shared_cache(22, kind, nkv, D, ps, kv, B)
    q = queries(c, B, rows, nkv * G)

    def call():
        status = ints([0])
        out = px().paged_attention(q, c.px, ints(kvs), causal=True, window=window, max_kv_len=kv, status=status)
        return out, status.item()

    want, status = call()
    assert status == 0 and torch.isfinite(want).all()
    first = [max(0, n - rows + 1 - window) // ps for n in kvs]
    assert any(f > 0 for f in first)
    assert any(max(0, n - rows + 1 - window) // tile * tile // ps < f for n, f in zip(kvs, first) for tile in (32, 64)), \
        "no tile begins in a page before the window"
    for gone in (-1, c.n_pages, 2 ** 31 - 1):
        for b, f in enumerate(first):
            c.table[b, :f] = gone
        got, status = call()
        assert status == 0 and torch.equal(got, want)
    c.table[0, first[0]] = -1
    got, status = call()
    assert status == px().PAGED_BAD_PAGE and got[0].isnan().any()
    if B > 1:
        assert torch.equal(got[1:], want[1:])


@pytest.mark.parametrize("kind,rows", [("bf16", 1), ("bf16", 60), ("f32", 1), ("f32", 60)])
def test_what_lies_before_the_window_may_be_anything(kind, rows):
    """The table's entry before the window names another request's page, or none, and what is
    read there is NaN: rows are what they are without it."""
    kv, window, ps = 170, 20, 16
    c = shared_cache(23, kind, 1, 64, ps, kv, 1)
    q = queries(c, 1, rows, 2)
    f = lambda: px().paged_attention(q, c.px, ints([kv]), window=window, max_kv_len=kv)  # noqa: E731
    want = host(f())
    first = (kv - rows + 1 - window) // ps
    assert first > 0
    page = int(c.host_table[0, first - 1])
    c.k[page], c.v[page] = float("nan"), float("inf")
    k, v = c.values()
    ref, mag = op.paged_attention(host(q), k, v, c.host_table, [kv], [rows], np.zeros(q.shape), window=window)
    bar = attention_bar(kind, host(q), np.where(np.isfinite(k), k, 0), ref, mag, 0.125, kv)
    check("named", host(f()), ref, bar)
    c.k[0], c.v[0] = float("nan"), float("inf")                # what a kernel reads instead of a number out of range
    c.table[0, :first] = -1
    check("not named", host(f()), ref, bar)
    check("before", want, ref, bar)


# (kind, head_dim, rows, K/V heads, heads of each, keys, split)
LAST = [("bf16", 64, 3, 1, 2, 61, False), ("bf16", 256, 1, 1, 8, 45, False), ("f32", 128, 2, 1, 4, 45, False),
        ("bf16", 128, 3, 1, 2, 701, True), ("f32", 64, 3, 1, 2, 701, True), ("bf16", 256, 3, 1, 2, 701, True),
        ("bf16", 64, 50, 1, 2, 145, False), ("f32", 64, 50, 1, 2, 61, False), ("f32", 256, 2, 1, 4, 61, False),
        ("bf16", 128, 50, 1, 2, 701, True), ("f32", 128, 50, 1, 2, 701, True), ("bf16", 256, 50, 1, 2, 701, True)]


@pytest.mark.parametrize("kind,D,rows,nkv,G,kv,split", LAST)
def test_an_infinite_value_of_the_last_token(kind, D, rows, nkv, G, kv, split):
    """The newest token, which ends inside a tile, has an infinite value in one dimension, minus
    infinity in another and NaN in a third: rows that see it have them, and the others none."""
    c = shared_cache(24, kind, nkv, D, 16, kv, 1)
    q = queries(c, 1, rows, nkv * G)
    assert (px().paged_attention_workspace(c.px, nkv * G, rows, kv) > 0) == split
    page, at = c.host_table[0, (kv - 1) // 16], (kv - 1) % 16
    for causal in (True, False):
        f = lambda: px().paged_attention(q, c.px, ints([kv]), max_kv_len=kv, causal=causal)  # noqa: E731
        c.v[page, at, 0, [5, 9, 11]] = 0.0
        want = f()
        c.v[page, at, 0, 5], c.v[page, at, 0, 9], c.v[page, at, 0, 11] = float("inf"), float("-inf"), float("nan")
        k, v = c.values()
        ref, mag = op.paged_attention(host(q), k, np.where(np.isfinite(v), v, 0), c.host_table, [kv], [rows],
                                      np.zeros(q.shape), causal=causal)
        bar = attention_bar(kind, host(q), k, ref, mag, D ** -0.5, kv)
        check("finite", host(want), ref, bar)
        got = f()
        see = [rows - 1] if causal else list(range(rows))
        hide = [t for t in range(rows) if t not in see]
        rest = [d for d in range(D) if d not in (5, 9, 11)]
        assert torch.isposinf(got[0, see, :, 5]).all() and torch.isneginf(got[0, see, :, 9]).all()
        assert got[0, see, :, 11].isnan().all()
        check("other dimensions", host(got)[..., rest], ref[..., rest], bar[..., rest])
        check("other rows", host(got)[:, hide], ref[:, hide], bar[:, hide])


def reference(c, q, kvs, causal=True, window=0):
    """(o, a, hit): attention over every request's keys in float64 with values that are not finite
    taken as 0, sum_j p_j |v_j|, and the rows that see a token holding such a value."""
    k, v = c.values()
    x = host(q)
    B, M, H, D = x.shape
    G = H // k.shape[2]
    o, mag, hit = np.zeros(x.shape), np.zeros(x.shape), np.zeros((B, M), dtype=bool)
    for b in range(B):
        n = kvs[b]
        if n == 0:
            continue
        kb, vb = op.tokens_of(k, c.host_table[b], n), op.tokens_of(v, c.host_table[b], n)
        odd = ~(np.isfinite(kb).all((1, 2)) & np.isfinite(vb).all((1, 2)))
        kb, vb = np.where(np.isfinite(kb), kb, 0.0), np.where(np.isfinite(vb), vb, 0.0)
        ok = op.visible(M, n, causal, window)
        hit[b] = (ok & odd).any(1)
        for h in range(H):
            s = np.where(ok, D ** -0.5 * (x[b, :, h] @ kb[:, h // G].T), -np.inf)
            p = np.exp(s - np.maximum(s.max(1, keepdims=True), -1e300))
            p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
            o[b, :, h], mag[b, :, h] = p @ vb[:, h // G], p @ np.abs(vb[:, h // G])
    return o, mag, hit


def put(c, token, x, heads=slice(None), dims=slice(3, None), pools=("k", "v")):
    """Value x in a token of the first request."""
    page, at = c.host_table[0, token // c.ps], token % c.ps
    for name in pools:
        pool = getattr(c, name)
        y = pool[page, at].float()
        y[heads, dims] = x
        z = y.to(pool.dtype)
        pool[page, at].view(torch.uint8 if c.kind == "fp8" else z.dtype).copy_(z.view(torch.uint8) if c.kind == "fp8" else z)


# (kind, head_dim, requests, rows, K/V heads, heads of each, keys, window, split)
PATHS = {
    # few rows: one wave a block (32 bits at head_dim 256 has the next shape)
    "few": [("bf16", 64, 1, 3, 1, 2, 61, 20, False), ("bf16", 128, 1, 3, 1, 2, 61, 20, False), ("bf16", 256, 1, 3, 1, 2, 61, 20, False),
            ("fp8", 64, 1, 3, 1, 2, 61, 20, False), ("fp8", 128, 2, 3, 2, 4, 61, 20, False), ("fp8", 256, 1, 1, 1, 8, 61, 10, False),
            ("f32", 64, 1, 3, 1, 2, 61, 20, False), ("f32", 128, 1, 3, 1, 2, 61, 20, False)],
    "few, many requests": [("bf16", 64, 512, 1, 8, 1, 97, 20, False), ("bf16", 128, 256, 1, 8, 1, 97, 20, False),
                           ("bf16", 256, 128, 1, 8, 1, 97, 20, False), ("fp8", 128, 256, 1, 8, 1, 97, 20, False),
                           ("f32", 128, 256, 1, 8, 1, 97, 20, False)],
    "few, split": [("bf16", 64, 1, 3, 1, 2, 2500, 1000, True), ("bf16", 128, 2, 3, 1, 2, 701, 0, True),
                   ("bf16", 256, 1, 3, 1, 2, 2500, 1000, True), ("fp8", 64, 1, 3, 1, 2, 701, 0, True),
                   ("fp8", 128, 1, 3, 2, 4, 2500, 1000, True), ("fp8", 256, 1, 3, 1, 2, 2500, 1000, True),
                   ("f32", 64, 1, 3, 1, 2, 701, 0, True), ("f32", 128, 1, 3, 1, 2, 2500, 1000, True)],
    "chunk": [("bf16", 64, 1, 50, 1, 2, 150, 40, False), ("bf16", 128, 2, 50, 1, 3, 150, 40, False),
              ("bf16", 256, 25, 9, 8, 1, 300, 70, False), ("fp8", 64, 1, 50, 1, 2, 150, 40, False),
              ("fp8", 128, 1, 50, 2, 4, 150, 40, False), ("fp8", 256, 1, 50, 1, 2, 150, 40, False),
              ("f32", 64, 1, 50, 1, 2, 61, 10, False), ("f32", 128, 1, 50, 1, 2, 61, 10, False), ("f32", 256, 1, 3, 1, 2, 61, 20, False)],
    "chunk, split": [("bf16", 64, 1, 50, 1, 2, 2500, 990, True), ("bf16", 128, 2, 50, 1, 3, 701, 0, True),
                     ("bf16", 256, 1, 300, 1, 8, 2500, 0, True), ("fp8", 64, 1, 50, 1, 2, 701, 0, True),
                     ("fp8", 128, 1, 50, 2, 4, 2500, 990, True), ("fp8", 256, 1, 50, 1, 2, 2500, 990, True),
                     ("f32", 64, 1, 50, 1, 2, 701, 0, True), ("f32", 128, 1, 50, 1, 2, 2500, 990, True),
                     ("f32", 256, 1, 50, 1, 2, 2500, 990, True)],
    # bf16 chunks of head_dim 256 in blocks of which a CU holds two
    "pairs": [("bf16", 256, 64, 9, 8, 1, 300, 70, False), ("bf16", 256, 33, 9, 8, 1, 61, 0, False)],
    "pairs, split": [("bf16", 256, 2, 150, 1, 2, 2500, 890, True), ("bf16", 256, 1, 50, 1, 2, 701, 0, True)],
}
ALL = [pytest.param(*p, id="-".join([name.replace(", ", "_").replace(" ", "_"), p[0]] + [str(x) for x in p[1:8]]))
       for name, ps in PATHS.items() for p in ps]
NAMES = "kind,D,B,rows,nkv,G,kv,window,split"


def set_up(seed, kind, D, B, rows, nkv, G, kv, split, ps=16):
    c = shared_cache(seed, kind, nkv, D, ps, kv, B)
    assert (px().paged_attention_workspace(c.px, nkv * G, rows, kv) > 0) == split, "another plan than the test means"
    return c, queries(c, B, rows, nkv * G)


@pytest.mark.parametrize(NAMES, ALL)
def test_lengths_at_the_edges_of_tiles(kind, D, B, rows, nkv, G, kv, window, split):
    """Every length near a multiple of 32 and of 64, one and none, causal and not, behind a
    window; the longest keeps the plan.  Two runs give the same bits."""
    c, q = set_up(31, kind, D, B, rows, nkv, G, kv, split)
    near = sorted({n for m in range(0, kv + 1, 32) for n in (m - 1, m, m + 1) if 0 <= n <= kv})
    near = near if len(near) <= 12 else near[:7] + near[-5:]
    for start in range(0, len(near), B):
        kvs = [near[(start + b) % len(near)] for b in range(B)]
        for causal, w in ((True, 0), (False, 0), (True, window)):
            f = lambda: px().paged_attention(q, c.px, ints(kvs), max_kv_len=kv, causal=causal, window=w)  # noqa: E731
            got = f()
            ref, mag, _ = reference(c, q, kvs, causal, w)
            k, _ = c.values()
            check(f"{kvs[:4]} causal {causal} window {w}", host(got), ref, attention_bar(kind, host(q), k, ref, mag, D ** -0.5, kv))
            assert torch.equal(got, f()), "two runs of one call differ"


@pytest.mark.parametrize(NAMES, ALL)
def test_hidden_nan_and_infinities_reach_no_row(kind, D, B, rows, nkv, G, kv, window, split):
    """NaN and infinities in the newest token, in one of the chunk and just before the window
    (in a tile that is read): rows that see none of them are what the formula gives without
    them, rows that do are not finite."""
    c, q = set_up(32, kind, D, B, rows, nkv, G, kv, split)
    odd = float("nan") if kind == "fp8" else float("inf")
    if rows > 1:
        put(c, kv - 1, odd)
        put(c, kv - rows + 2, float("nan"))
    if window:
        lo = kv - rows + 1 - window
        assert (lo - 1) // 32 == lo // 32, "the token before the window lies in another tile"
        put(c, lo - 1, odd, pools=("v",))
    kvs = [kv] * B
    got = host(px().paged_attention(q, c.px, ints(kvs), max_kv_len=kv, window=window))
    ref, mag, hit = reference(c, q, kvs, True, window)
    assert not hit.all() and (rows == 1 or hit.any())
    k, _ = c.values()
    bar = attention_bar(kind, host(q), np.where(np.isfinite(k), k, 0), ref, mag, D ** -0.5, kv)
    check("rows that see none", got[~hit], ref[~hit], bar[~hit])
    assert not np.isfinite(got[hit]).all(-1).any()


@pytest.mark.parametrize(NAMES, ALL)
def test_what_rows_see_stays_what_it_is(kind, D, B, rows, nkv, G, kv, window, split):
    """An infinite value (8 bits: NaN alone, they have no infinity) and a NaN in the first token,
    which every row sees: those dimensions are infinite and NaN, the others what they were."""
    c, q = set_up(33, kind, D, B, rows, nkv, G, kv, split)
    put(c, 0, 0.0, dims=[5, 9], pools=("v",))
    f = lambda: px().paged_attention(q, c.px, ints([kv] * B), max_kv_len=kv)  # noqa: E731
    want = f()
    put(c, 0, float("nan"), dims=9, pools=("v",))
    if kind != "fp8":
        put(c, 0, float("inf"), dims=5, pools=("v",))
    got = f()
    assert got[..., 9].isnan().all()
    if kind != "fp8":
        assert torch.isposinf(got[..., 5]).all()
    rest = [d for d in range(D) if d not in (5, 9)]
    assert torch.equal(got[..., rest], want[..., rest])


@pytest.mark.parametrize(NAMES, ALL)
def test_bad_pages_and_lengths(kind, D, B, rows, nkv, G, kv, window, split):
    """A page or a length out of range: that request becomes NaN and raises the bit, the
    others keep their bits."""
    c, q = set_up(34, kind, D, B, rows, nkv, G, kv, split)
    bad = B - 1

    def call(kvs, new=None):
        status = ints([0])
        out = px().paged_attention(q, c.px, ints(kvs), new_len=None if new is None else ints(new), max_kv_len=kv, causal=False,
                                   status=status)
        return out, status.item()

    want, status = call([kv] * B)
    assert status == 0 and torch.isfinite(want).all()
    last = (kv - 1) // c.ps
    for at, page in ((0, -1), (last, c.n_pages), (last // 2, -2 ** 31)):
        c.table.copy_(torch.from_numpy(c.host_table))
        c.table[bad, at] = page
        got, status = call([kv] * B)
        assert status == px().PAGED_BAD_PAGE and got[bad].isnan().all() and torch.equal(got[:bad], want[:bad])
    c.table.copy_(torch.from_numpy(c.host_table))
    for n, new in ((kv + 1, None), (-1, None), (kv, rows + 1)):
        got, status = call([kv] * bad + [n], None if new is None else [rows] * bad + [new])
        assert status == px().PAGED_BAD_LENGTH and got[bad].isnan().all() and torch.equal(got[:bad], want[:bad])
