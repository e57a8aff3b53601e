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
