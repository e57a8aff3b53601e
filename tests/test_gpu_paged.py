"""The paged key/value cache on the GPU against the float64 oracle.

Bars, element by element, from the arithmetic (u = 2^-24, the half step of float32;
h = 2^-8, that of bfloat16, each relative to the value):
  attention  A score is a 32-bit sum of D products, off by (D + 2) u times the sum of
             their magnitudes; twice the largest such error, e, bounds the relative
             error of a weight (numerator and sum), the exponential adds a few u, the
             sums over n keys n u.  With m = sum_j p_j |v_j|:
               f32        (2 e + (n + 32) u) m
               bf16, fp8  the same, plus h m for the weights' rounding and h |o| for
                          the output's
  norm       the sum of squares is off by (D + 4) u, its root by half of that; gain,
             rotation and angle (2^-25 of a turn, 3.2 u) add 16 u: ((D + 4) / 2 + 16) u (|a| + |b|)
             over the pair, plus h |y| for bf16
  append     values are stored exactly; rotated keys 16 u (|a| + |b|), plus h |y| for bf16;
             8 bits: half a step of the code (2^-4 of the value, 2^-10 below the
             normal range) of value / scale, with u for the quotient
  gather     exact; 8 bits: the float32 product rounded once, exact
"""
import math

import numpy as np
import pytest

import oracle.paged as op
from oracle.numerics import E4M3FN_TABLE, rope

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U, H16 = 2.0 ** -24, 2.0 ** -8
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
SENTINEL = 7.25


def px():
    import paper_2608_03682_amd as m
    return m


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def host(t):
    """Device values as float64; 8-bit codes decoded by the oracle's table."""
    if t.dtype == torch.float8_e4m3fn:
        return E4M3FN_TABLE[t.view(torch.uint8).cpu().numpy()]
    return t.cpu().double().numpy()


class Cache:
    """Pools of random values in random pages, NaN in every row that no request owns,
    with the oracle's view of them."""

    def __init__(self, seed, kind, nkv, D, ps, lens, heads_first=False, layers=0, spare=2, stale=True):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.nkv, self.D, self.ps, self.lens = kind, nkv, D, ps, lens
        need = [-(-n // ps) for n in lens]
        self.n_pages = max(1, sum(need) + spare)
        order = torch.randperm(self.n_pages, generator=g).tolist()
        table = np.full((len(lens), max(1, max(need))), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.host_table, self.table = table, torch.from_numpy(table).cuda()
        lead = (layers,) if layers else ()
        shape = lead + ((self.n_pages, nkv, ps, D) if heads_first else (self.n_pages, ps, nkv, D))
        self.ks = self.vs = None
        if kind == "fp8":
            self.ks, self.vs = 0.02 + 0.03 * torch.rand(nkv, generator=g), 0.02 + 0.03 * torch.rand(nkv, generator=g)
        owned = torch.zeros(self.n_pages, ps, dtype=torch.bool)
        for b, n in enumerate(lens):
            for p in range(n):
                owned[table[b, p // ps], p % ps] = True

        def pool(scale, offset):
            x = torch.randn(lead + (self.n_pages, ps, nkv, D), generator=g) + offset * torch.randn(nkv, D, generator=g)
            if kind == "fp8":
                x = (x / scale[:, None]).clamp(-448, 448)
            if stale:
                x = torch.where(owned[..., None, None], x, float("nan"))
            x = x.to(TORCH[kind])
            raw = torch.empty(shape, dtype=TORCH[kind])
            y = raw.transpose(-3, -2) if heads_first else raw
            y.view(torch.uint8 if kind == "fp8" else y.dtype).copy_(x.view(torch.uint8) if kind == "fp8" else x)
            d = raw.cuda()
            return d.transpose(-3, -2) if heads_first else d

        self.k, self.v = pool(self.ks, 0.3), pool(self.vs, 0.5)
        self.dks = None if self.ks is None else self.ks.cuda()
        self.dvs = None if self.vs is None else self.vs.cuda()
        self.px = px().PagedCache(self.k, self.v, self.table, self.dks, self.dvs)

    def values(self):
        k, v = host(self.k), host(self.v)
        if self.kind == "fp8":
            k, v = k * self.ks.double().numpy()[:, None], v * self.vs.double().numpy()[:, None]
        return k, v


def attention_bar(kind, q, k, o, mag, scale, n):
    kmax = np.abs(np.nan_to_num(k)).max((0, 1))                      # [nkv][D]
    G = q.shape[2] // k.shape[2]
    reach = scale * (np.abs(q) * np.repeat(kmax, G, 0)).sum(-1)      # sum of magnitudes, at most
    e = (q.shape[3] + 2) * U * reach[..., None]
    bar = (2 * e + (n + 32) * U) * mag
    return bar if kind == "f32" else bar + H16 * mag + H16 * np.abs(o) * (1 + H16)


def check(name, got, ref, bar):
    err = np.abs(got - ref)
    worst = float((err / np.maximum(bar, 1e-300)).max()) if err.size else 0.0
    print(f"[parity] {name}: max_abs={err.max() if err.size else 0:.3e}, {worst:.2f} of its bar", flush=True)
    assert np.isfinite(got).all(), f"{name}: non-finite output"
    assert (err <= bar).all(), f"{name}: {worst:.2f} times its bar"


def run_attention(name, c, rows, H, new, kv, causal=True, window=0, seed=5, q=None, **kw):
    dt = torch.float32 if c.kind == "f32" else torch.bfloat16
    if q is None:
        q = (1.5 * torch.randn(len(kv), rows, H, c.D, generator=torch.Generator().manual_seed(seed))).to(dt).cuda()
    out = torch.full(q.shape, SENTINEL, dtype=dt, device="cuda")
    status = ints([0])
    got = px().paged_attention(q, c.px, ints(kv), new_len=ints(new), causal=causal, window=window, out=out,
                               status=status, **kw)
    torch.cuda.synchronize()
    assert got is out and status.item() == 0
    k, v = c.values()
    ref, mag = op.paged_attention(host(q), k, v, c.host_table, kv, new, np.full(q.shape, SENTINEL), causal=causal,
                                  window=window)
    got = host(out)
    for b, m in enumerate(new):
        assert (got[b, m:] == SENTINEL).all(), "rows behind the last were written"
    check(name, got, ref, attention_bar(c.kind, host(q), k, ref, mag, c.D ** -0.5, max(kv)))
    return out


KINDS = ["bf16", "fp8", "f32"]
DIMS = [64, 128, 256]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("kind", KINDS)
def test_single_tokens_at_the_edges_of_tiles_and_pages(kind, D):
    kv = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 300]
    c = Cache(1, kind, 2, D, 16, kv)
    run_attention(f"tokens {kind} {D}", c, 1, 6, [1] * len(kv), kv)
    run_attention(f"tokens {kind} {D}, keys not split", c, 1, 6, [1] * len(kv), kv, max_kv_len=300)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("kind", KINDS)
def test_chunks_ragged_and_causal(kind, D):
    # 70 rows x 3 heads: two row tiles of a K/V head; new_len 0, fewer keys than rows
    kv, new = [131, 70, 64, 20, 0, 257], [70, 70, 1, 33, 5, 0]
    c = Cache(2, kind, 1, D, 32, kv, heads_first=True)
    run_attention(f"chunk {kind} {D}", c, 70, 3, new, kv)


@pytest.mark.parametrize("kind,rows,causal,window", [
    ("bf16", 45, False, 0), ("bf16", 45, True, 1), ("bf16", 45, True, 40), ("bf16", 3, True, 33), ("bf16", 3, False, 0),
    ("fp8", 45, True, 100), ("fp8", 2, True, 17), ("f32", 45, False, 0), ("f32", 45, True, 40), ("f32", 4, True, 1)])
def test_masks(kind, rows, causal, window):
    kv, new = [200, 97, 45, 30], [rows, max(1, rows - 7), rows, 1]
    c = Cache(3, kind, 2, 128 if rows > 40 else 64, 64, kv)
    run_attention(f"mask {kind} {rows} {causal} {window}", c, rows, 8, new, kv, causal=causal, window=window)


@pytest.mark.parametrize("B,rows,nkv,kv_max,ps,causal,window", [
    (33, 9, 8, 40, 16, True, 0),        # more blocks than CUs: two of a CU
    (25, 9, 8, 300, 16, False, 0),      # about a block for every CU, keys not split
    (25, 9, 8, 300, 64, True, 70),
    (2, 150, 1, 2500, 16, True, 0),     # few blocks: keys split
    (2, 150, 1, 2500, 64, True, 900),   # the same behind a window, in the workspace sized without it
    (1, 300, 1, 300, 4096, False, 0)])
def test_chunks_of_head_dim_256(B, rows, nkv, kv_max, ps, causal, window):
    kv = [kv_max - 7 * b for b in range(B)]
    new = [max(0, min(rows, kv[b]) - b) for b in range(B)]
    c = Cache(11, "bf16", nkv, 256, ps, [max(0, n) for n in kv])
    kv = [max(0, n) for n in kv]
    new = [min(m, n) for m, n in zip(new, kv)]
    H = nkv * (1 if nkv == 8 else 2)
    size = px().paged_attention_workspace(c.px, H, rows, kv_max)
    ws = torch.full((max(16, size),), 0x7f, dtype=torch.uint8, device="cuda")
    a = run_attention(f"256 {B} {rows}", c, rows, H, new, kv, causal=causal, window=window, max_kv_len=kv_max, workspace=ws)
    b = run_attention("again", c, rows, H, new, kv, causal=causal, window=window, max_kv_len=kv_max, workspace=ws)
    assert torch.equal(a, b), "two runs of one call differ"


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_keys_split_over_blocks(kind, rows, D):
    kv = [2500, 90, 1]
    c = Cache(4, kind, 1, D, 64, kv)
    assert px().paged_attention_workspace(c.px, 4, rows) > 0
    new = [min(rows, n) for n in kv]
    a = run_attention(f"split {kind} {rows} {D}", c, rows, 4, new, kv)
    b = run_attention("again", c, rows, 4, new, kv)
    assert torch.equal(a, b), "two runs of one call differ"


@pytest.mark.parametrize("rows", [4, 60])
@pytest.mark.parametrize("kind", KINDS)
def test_what_a_row_does_not_see_does_not_reach_it(kind, rows):
    """NaN and infinities in later tokens (and, with a window, in earlier ones): rows that
    see none of them are what they are without them; rows that do are not finite."""
    kv, D = [150], 64
    c = Cache(6, kind, 1, D, 32, kv)
    clean = host(run_attention("clean", c, rows, 2, [rows], kv, window=50))
    bad = {150 - rows + 2: float("nan"), 149: float("inf") if kind != "fp8" else float("nan"), 60: float("nan")}
    for p, x in bad.items():
        page, at = c.host_table[0, p // 32], p % 32
        for pool in (c.k, c.v):
            y = pool[page, at].float()
            y[:, 3:] = x
            pool[page, at] = y.to(pool.dtype)
    q = (1.5 * torch.randn(1, rows, 2, D, generator=torch.Generator().manual_seed(5))).to(
        torch.float32 if kind == "f32" else torch.bfloat16).cuda()
    for max_kv in (150, None):
        got = host(px().paged_attention(q, c.px, ints(kv), causal=True, window=50, max_kv_len=max_kv))
        ok = op.visible(rows, 150, True, 50)
        for t in range(rows):
            hit = any(ok[t, p] for p in bad)
            if hit:
                assert not np.isfinite(got[0, t]).all(), t
            else:
                k, v = c.values()
                ref, mag = op.paged_attention(host(q), k, v, c.host_table, kv, [rows], np.zeros(q.shape), window=50)
                bar = attention_bar(kind, host(q), np.where(np.isfinite(k), k, 0), ref, mag, D ** -0.5, 150)
                assert (np.abs(got[0, t] - ref[0, t]) <= bar[0, t]).all(), t
    assert np.isfinite(clean).all()


@pytest.mark.parametrize("rows", [3, 50])
def test_a_value_that_rows_see_stays_what_it_is(rows):
    """An infinite and a NaN value in a token that every row sees: those dimensions are
    infinite and NaN, the others what they are without them (both shapes, split and not)."""
    D, kv = 128, [700]
    c = Cache(18, "bf16", 1, D, 16, kv)
    q = (1.5 * torch.randn(1, rows, 4, D, generator=torch.Generator().manual_seed(5))).bfloat16().cuda()
    page, at = c.host_table[0, 100 // 16], 100 % 16
    for max_kv in (700, None):
        c.v[page, at, 0, 5], c.v[page, at, 0, 9] = 0.0, 0.0
        want = px().paged_attention(q, c.px, ints(kv), max_kv_len=max_kv)
        c.v[page, at, 0, 5], c.v[page, at, 0, 9] = float("inf"), float("nan")
        got = px().paged_attention(q, c.px, ints(kv), max_kv_len=max_kv)
        rest = [d for d in range(D) if d not in (5, 9)]
        assert torch.isposinf(got[..., 5]).all() and got[..., 9].isnan().all()
        assert torch.equal(got[..., rest], want[..., rest])


@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_a_key_are_zero_beside_infinite_values(kind):
    """More rows than keys: the first rows see none, and NaN in the keys that the others
    see does not reach them."""
    for rows, heads in ((6, 2), (60, 3)):
        c = Cache(19, kind, 1, 64, 16, [5, 20])
        for b, p in ((0, 4), (1, 19)):
            page = c.host_table[b, p // 16]
            y = c.v[page, p % 16].float()
            y[:, 7] = float("nan")
            c.v[page, p % 16] = y.to(c.v.dtype)
        q = torch.ones(2, rows, heads, 64, device="cuda", dtype=torch.float32 if kind == "f32" else torch.bfloat16)
        for max_kv in (20, None):
            got = px().paged_attention(q, c.px, ints([5, 20]), max_kv_len=max_kv)
            for b, n in enumerate((5, 20)):
                if rows > n:
                    assert (got[b, :rows - n] == 0).all()
                last = got[b, rows - 1]
                assert last[:, 7].isnan().all() and torch.isfinite(last[:, :7]).all() and torch.isfinite(last[:, 8:]).all()
                if n > 1:                            # the row before the last does not see the NaN
                    assert torch.isfinite(got[b, rows - 2]).all()


def test_large_scores_and_zero_scales():
    """Scores of thousands (one key takes all), and an 8-bit cache whose keys have scale 0."""
    c = Cache(7, "f32", 1, 64, 16, [90])
    q = 400.0 * torch.randn(1, 2, 1, 64, generator=torch.Generator().manual_seed(1)).cuda()
    run_attention("large scores", c, 2, 1, [2], [90], q=q)
    c = Cache(8, "fp8", 1, 64, 16, [70])
    c.dks.zero_()
    c.ks.zero_()
    run_attention("zero scale", c, 3, 2, [3], [70])


def test_strides_of_a_projected_row_and_other_layers():
    """Queries as a slice of [q | k | v] rows, output into a wider buffer, the second of
    three layers, a table with a row stride, single heads and single requests."""
    c = Cache(9, "bf16", 2, 64, 16, [77, 50], layers=3)
    wide = torch.randn(2, 5, 4 + 2 + 2, 64, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    q = wide[:, :, :4]
    out = torch.full((2, 5, 12, 64), SENTINEL, dtype=torch.bfloat16, device="cuda")
    table = torch.full((2, 9), -5, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    pc = px().PagedCache(c.k, c.v, table[:, :c.table.shape[1]])
    px().paged_attention(q, pc, ints([77, 50]), layer=1, out=out[:, :, 3:7])
    k, v = c.values()
    ref, mag = op.paged_attention(host(q), k[1], v[1], c.host_table, [77, 50], [5, 5], np.zeros(q.shape))
    check("strided", host(out[:, :, 3:7]), ref, attention_bar("bf16", host(q), k[1], ref, mag, 0.125, 77))
    assert (out[:, :, :3] == SENTINEL).all() and (out[:, :, 7:] == SENTINEL).all()


def test_offsets_beyond_32_bits():
    """Pages that lie more than 4 GiB into their pool."""
    ps, D, n_pages = 64, 128, 300000                          # 4.9 GB a pool
    k = torch.empty(n_pages, ps, 1, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = np.array([[n_pages - 1, 3, n_pages - 2]], dtype=np.int32)
    kn = torch.randn(1, 150, 1, D, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    vn = torch.randn(1, 150, 1, D, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    pc = px().PagedCache(k, v, torch.from_numpy(table).cuda())
    px().paged_append(pc, kn, vn, ints([0]))
    assert torch.equal(k[n_pages - 1], kn[0, :64]) and torch.equal(v[n_pages - 2, :22], vn[0, 128:])
    g = px().paged_gather(pc, ints([150]), 150)
    assert torch.equal(g[0, 0, 0], kn[0, :, 0]) and torch.equal(g[0, 1, 0], vn[0, :, 0])
    for rows in (2, 50):
        q = torch.randn(1, rows, 4, D, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
        got = host(px().paged_attention(q, pc, ints([150])))
        kp, vp = host(kn[0])[None], host(vn[0])[None]
        ref, mag = op.paged_attention(host(q), kp, vp, [[0]], [150], [rows], np.zeros(q.shape))
        check(f"far pages, {rows} rows", got, ref, attention_bar("bf16", host(q), kp, ref, mag, D ** -0.5, 150))


def test_bad_pages_and_lengths_become_nan_and_status():
    kv = [100, 100, 100]
    for kind in KINDS:
        for rows in (1, 70):
            c = Cache(10, kind, 1, 64, 32, kv)
            good = host(px().paged_attention(torch.ones(3, rows, 2, 64, device="cuda", dtype=torch.float32 if kind == "f32" else torch.bfloat16), c.px, ints(kv)))
            for page in (-1, c.n_pages, 2 ** 31 - 1, -2 ** 31):
                c.table.copy_(torch.from_numpy(c.host_table))
                c.table[1, 0] = page
                status = ints([0])
                q = torch.ones(3, rows, 2, 64, device="cuda", dtype=torch.float32 if kind == "f32" else torch.bfloat16)
                got = host(px().paged_attention(q, c.px, ints(kv), status=status))
                assert status.item() == px().PAGED_BAD_PAGE
                assert np.isnan(got[1]).all() and (got[[0, 2]] == good[[0, 2]]).all()
            c.table.copy_(torch.from_numpy(c.host_table))
            for lens, new in (([100, 129, 100], None), ([100, -1, 100], None), ([100, 100, 100], [rows, rows + 1, rows])):
                status = ints([0])
                got = host(px().paged_attention(q, c.px, ints(lens), new_len=None if new is None else ints(new),
                                                status=status))
                assert status.item() == px().PAGED_BAD_LENGTH
                assert np.isnan(got[1]).all() and (got[[0, 2]] == good[[0, 2]]).all()


# ---------------------------------------------------------------------------
# norms and rotation
# ---------------------------------------------------------------------------
def pair_sum(x, D):
    return np.abs(x[..., :D // 2]) + np.abs(x[..., D // 2:])


def turn_bar(y, D, steps, bf16):
    m = pair_sum(y, D)
    bar = steps * U * np.concatenate([m, m], -1)
    return bar + (H16 * np.abs(y) * (1 + H16) if bf16 else 0.0) + 1e-37


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3, 5, 4, 1), (1, 1, 1, 1), (2, 37, 5, 2), (1100, 3, 2, 2)])
def test_norm_rope(shape, kind, D):
    B, M, nq, nk = shape
    g = torch.Generator().manual_seed(B + D)
    row = (2.0 * torch.randn(B, M, nq + nk, D, generator=g)).to(TORCH[kind]).cuda()
    q, k = row[:, :, :nq], row[:, :, nq:]
    qg, kg = (0.2 * torch.randn(D, generator=g)).cuda(), (0.2 * torch.randn(D, generator=g)).cuda()
    past = [[0, 1, 1 << 20, 2 ** 31 - 1 - M][b % 4] for b in range(B)]
    new = [max(0, M - b % 3) for b in range(B)]
    qo, ko = torch.full(q.shape, SENTINEL, dtype=q.dtype, device="cuda"), torch.full(k.shape, SENTINEL, dtype=q.dtype, device="cuda")
    for eps, base, gains in ((1e-6, 1e4, True), (1e-5, 0.0, False), (0.0, 1e6, False), (1e-6, 1.0, True)):
        gq, gk = (qg, kg) if gains else (None, None)
        status = ints([0])
        px().qk_norm_rope(q, k, gq, gk, eps=eps, rope_base=base, past_len=ints(past), new_len=ints(new), q_out=qo,
                          k_out=ko, status=status)
        assert status.item() == 0
        for x, gain, o in ((q, gq, qo), (k, gk, ko)):
            ref = op.qk_norm_rope(host(x), None if gain is None else host(gain), eps, base, past, new,
                                  np.full(x.shape, SENTINEL))
            check(f"norm_rope {shape} {kind} {D} {eps} {base}", host(o), ref,
                  turn_bar(ref, D, ((D + 4) / 2 if eps else 0) + 16, kind == "bf16"))


def test_norm_rope_in_place_queries_alone_and_refusals():
    q = torch.randn(2, 3, 2, 64, generator=torch.Generator().manual_seed(1)).cuda()
    want, none = px().qk_norm_rope(q)
    assert none is None
    x = q.clone()
    px().qk_norm_rope(x, q_out=x)
    assert torch.equal(x, want)
    # a length out of range: the request is left as it was
    x = q.clone()
    status = ints([0])
    px().qk_norm_rope(x, q_out=x, new_len=ints([4, 3]), past_len=ints([0, 0]), status=status)
    assert status.item() == px().PAGED_BAD_LENGTH and torch.equal(x[0], q[0]) and not torch.equal(x[1], q[1])
    x = q.clone()
    px().qk_norm_rope(x, q_out=x, past_len=ints([-1, 0]), status=status)
    assert torch.equal(x[0], q[0]) and torch.equal(x[1], want[1])
    # zero rows give zeros, not NaN
    assert (px().qk_norm_rope(torch.zeros(1, 1, 1, 64, device="cuda"))[0] == 0).all()
    for bad in (dict(q_out=q[:, :2]), dict(past_len=ints([0])), dict(new_len=torch.zeros(2, device="cuda")),
                dict(q_gain=torch.zeros(32, device="cuda")), dict(status=torch.zeros(1, device="cuda")), dict(k_out=q)):
        with pytest.raises(ValueError):
            px().qk_norm_rope(q, **bad)
    with pytest.raises(ValueError):
        px().qk_norm_rope(q.transpose(2, 3))
    with pytest.raises(ValueError):
        px().qk_norm_rope(q.cpu())
    assert px().qk_norm_rope(q[:0])[0].shape == (0, 3, 2, 64)


# ---------------------------------------------------------------------------
# append and gather
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads_first", [False, True])
def test_append_and_gather(kind, D, heads_first):
    past, new, M = [0, 15, 100, 31, 7], [20, 1, 33, 0, 33], 33
    lens = [p + n for p, n in zip(past, new)]
    c = Cache(11, kind, 3, D, 16, lens, heads_first, stale=False)
    k0, v0 = host(c.k), host(c.v)
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    row = torch.randn(5, M, 6, D, generator=torch.Generator().manual_seed(D)).to(dt).cuda()
    row[0, 0, 3, 0] = 40.0                                    # saturates the 8-bit cache
    kn, vn = row[:, :, :3], row[:, :, 3:]
    for base in (0.0, 1e4):
        status = ints([0])
        px().paged_append(c.px, kn, vn, ints(past), new_len=ints(new), rope_base=base, status=status)
        assert status.item() == 0
        for pool, x, start, b, s in ((c.k, kn, k0, base, c.ks), (c.v, vn, v0, 0.0, c.vs)):
            ref = op.paged_append(start, c.host_table, host(x), past, new, b)
            marks = op.paged_append(np.zeros_like(start), c.host_table, np.ones(x.shape), past, new) > 0
            if b > 0:
                tol = op.paged_append(np.zeros_like(start), c.host_table, np.concatenate(
                    [pair_sum(host(x), D)] * 2, -1), past, new) * 16 * U
            else:
                tol = np.zeros_like(start)
            got = host(pool)
            assert (got[~marks] == start[~marks]).all(), "rows that are not new were written"
            if kind == "fp8":
                sc = s.double().numpy()[:, None]
                want = np.clip(ref / sc, -448, 448)
                want = np.where(marks, want, start)
                bar = np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10) * (1 + 4 * U) + (tol / sc + np.abs(want) * 2 * U)
                assert (np.abs(got - want)[marks] <= bar[marks]).all()
                if s is c.vs:
                    assert np.abs(got).max() == 448.0
            elif b == 0:
                assert (got == ref).all()
            else:
                bar = tol + (H16 * np.abs(ref) * (1 + H16) if kind == "bf16" else 0.0)
                assert (np.abs(got - ref)[marks] <= bar[marks]).all()
    g = px().paged_gather(c.px, ints(lens), 140)
    k, v = host(c.k), host(c.v)
    if kind == "fp8":
        f = lambda p, s: (p.astype(np.float32) * s.numpy()[:, None]).astype(np.float32)  # noqa: E731
        k, v = f(k, c.ks), f(v, c.vs)
    ref = torch.from_numpy(op.paged_gather(k, v, c.host_table, lens, 140)).to(dt)
    assert torch.equal(g[0].cpu(), ref)


def test_append_and_gather_skip_what_is_out_of_range():
    c = Cache(12, "bf16", 1, 64, 16, [32, 32, 32, 32], stale=False)
    before_k, before_v = c.k.clone(), c.v.clone()
    x = torch.randn(4, 8, 1, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    status = ints([0])
    # past the table's room, negative lengths, more rows than there are: nothing of theirs is written
    px().paged_append(c.px, x, x, ints([25, -1, 0, 24]), new_len=ints([8, 4, 9, -3]), status=status)
    assert status.item() == px().PAGED_BAD_LENGTH
    assert torch.equal(c.k, before_k) and torch.equal(c.v, before_v)
    # a bad page: its tokens alone are left out
    status.zero_()
    c.table[0, 1] = c.n_pages
    c.table[1, 0] = -7
    px().paged_append(c.px, x, x, ints([12, 12, 12, 12]), status=status)
    assert status.item() == px().PAGED_BAD_PAGE
    t = c.host_table
    assert torch.equal(c.k[t[0, 0], 12:], x[0, :4]) and torch.equal(c.k[t[0, 1]], before_k[t[0, 1]])
    assert torch.equal(c.v[t[1, 1], :4], x[1, 4:]) and torch.equal(c.v[t[1, 0]], before_v[t[1, 0]])
    assert torch.equal(c.k[t[3, 0], 12:], x[3, :4]) and torch.equal(c.k[t[3, 1], :4], x[3, 4:])
    status.zero_()
    g = px().paged_gather(c.px, ints([32, 33, 20, -1]), 32, status=status)
    assert status.item() == px().PAGED_BAD_PAGE | px().PAGED_BAD_LENGTH
    assert g[0, :, 0, 16:].isnan().all() and g[0, 0, 0, :16].equal(c.k[t[0, 0], :, 0])
    assert g[0, :, 1].isnan().all() and g[0, :, 3].isnan().all() and (g[0, :, 2, 20:] == 0).all()


def test_a_scale_of_zero_holds_zeros():
    """A head of zeros whose scale is its largest magnitude / 448: codes of 0, not of 0 / 0; NaN stays NaN."""
    D, nkv, ps = 128, 2, 16
    pools = torch.full((2, 2, ps, nkv, D), 0x55, dtype=torch.uint8, device="cuda")
    k_scale, v_scale = torch.tensor([0.0, 0.5], device="cuda"), torch.tensor([0.5, 0.0], device="cuda")
    c = px().PagedCache(pools[0], pools[1], ints([[1]]), k_scale, v_scale)
    k, v = torch.zeros(2, 1, 3, nkv, D, dtype=torch.bfloat16, device="cuda")
    k[0, 2, 0, 5] = float("nan")
    for base in (0.0, 1e4):
        px().paged_append(c, k, v, ints([0]), rope_base=base)
        got = pools[:, 1, :3].cpu()
        for pool in (0, 1):
            assert ((got[pool, :2] & 0x7f) == 0).all()
        assert (got[0, 2, 0, 5] & 0x7f) == 0x7f and ((got[1, 2] & 0x7f) == 0).all()
    out = px().paged_gather(c, ints([2]), 2)
    assert (out == 0).all()
    q = torch.ones(1, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    assert (px().paged_attention(q, c, ints([2])) == 0).all()


def test_a_shared_page_and_the_same_request_twice():
    """Two requests read the pages of one prefix; equal requests have equal results."""
    c = Cache(13, "bf16", 2, 128, 16, [64, 64, 64])
    c.table[1, :3] = c.table[0, :3]
    c.table[2] = c.table[0]
    c.host_table[:] = c.table.cpu().numpy()
    q = torch.randn(1, 7, 4, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda().expand(3, -1, -1, -1)
    out = run_attention("shared", c, 7, 4, [7, 7, 7], [60, 64, 60], q=q)
    assert torch.equal(out[0], out[2])


# ---------------------------------------------------------------------------
# as a program uses them
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", KINDS)
def test_a_prompt_in_chunks_is_the_prompt_at_once(kind):
    """norm + rotation, append and attention over chunks of 1 to 40 tokens, then the
    gather: each step against the oracle on the values the step before left."""
    nq, nkv, D, ps, total = 4, 2, 64, 16, 90
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(21)
    c = Cache(14, kind, nkv, D, ps, [total, total - 13], stale=True)
    gain = (0.1 * torch.randn(D, generator=g)).cuda()
    chunks = [(0, 40), (40, 1), (41, 33), (74, 16)]
    for at, m in chunks:
        row = torch.randn(2, m, nq + 2 * nkv, D, generator=g).to(dt).cuda()
        past = [at, max(0, at - 13)]
        new = [m, m if at else m - 13]
        pl, nl = ints(past), ints(new)
        q, k = px().qk_norm_rope(row[:, :, :nq], row[:, :, nq:nq + nkv], gain, gain, past_len=pl, new_len=nl,
                                 q_out=torch.zeros(2, m, nq, D, dtype=dt, device="cuda"),
                                 k_out=torch.zeros(2, m, nkv, D, dtype=dt, device="cuda"))
        for x, y in ((row[:, :, :nq], q), (row[:, :, nq:nq + nkv], k)):
            ref = op.qk_norm_rope(host(x), host(gain), 1e-6, 1e4, past, new, np.zeros(x.shape))
            check(f"chunk at {at}: norm", host(y), ref, turn_bar(ref, D, (D + 4) / 2 + 16, kind != "f32"))
        px().paged_append(c.px, k, row[:, :, nq + nkv:], pl, new_len=nl)
        kv = [p + n for p, n in zip(past, new)]
        run_attention(f"chunk at {at}: attention", c, m, nq, new, kv, q=q)
    got = px().paged_gather(c.px, ints([total, total - 13]), total)
    k, v = c.values()
    ref = op.paged_gather(k, v, c.host_table, [total, total - 13], total)
    assert np.isfinite(host(got)).all()
    assert (np.abs(host(got[0]) - ref) <= (H16 if kind == "fp8" else 0) * np.abs(ref)).all()


def test_captured_calls_serve_later_lengths():
    """Two captured graphs of a token step, each with a workspace of its own, replayed in
    turn with other lengths, tables and values, with eager work between."""
    kvmax, D, nq, nkv = 900, 128, 8, 2
    c = Cache(15, "bf16", nkv, D, 16, [kvmax, kvmax, 500], stale=False)
    kv, past = ints([1, 1, 1]), ints([0, 0, 0])
    row = torch.zeros(3, 1, nq + 2 * nkv, D, dtype=torch.bfloat16, device="cuda")
    bufs = []
    for _ in range(2):
        bufs.append(dict(ws=torch.empty(px().paged_attention_workspace(c.px, nq, 1, kvmax), dtype=torch.uint8, device="cuda"),
                         q=torch.zeros(3, 1, nq, D, dtype=torch.bfloat16, device="cuda"),
                         k=torch.zeros(3, 1, nkv, D, dtype=torch.bfloat16, device="cuda"),
                         out=torch.zeros(3, 1, nq, D, dtype=torch.bfloat16, device="cuda")))

    def step(b):
        px().qk_norm_rope(row[:, :, :nq], row[:, :, nq:nq + nkv], past_len=past, q_out=b["q"], k_out=b["k"])
        px().paged_append(c.px, b["k"], row[:, :, nq + nkv:], past)
        px().paged_attention(b["q"], c.px, kv, max_kv_len=kvmax, out=b["out"], workspace=b["ws"])

    graphs = []
    for b in bufs:
        step(b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(b)
        graphs.append(g)
    gen = torch.Generator().manual_seed(9)
    eager = dict(ws=torch.empty_like(bufs[0]["ws"]), q=torch.zeros_like(bufs[0]["q"]), k=torch.zeros_like(bufs[0]["k"]),
                 out=torch.zeros_like(bufs[0]["out"]))
    for i, n in enumerate([5, 900, 64, 333, 17, 899]):
        row.copy_(torch.randn(row.shape, generator=gen).bfloat16())
        lens = [n, max(1, n // 2), min(500, n)]
        kv.copy_(ints(lens))
        past.copy_(ints([x - 1 for x in lens]))
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for b in bufs:
            assert torch.equal(b["out"], eager["out"]) and torch.equal(b["k"], eager["k"])
        k, v = c.values()
        ref, mag = op.paged_attention(host(eager["q"]), k, v, c.host_table, lens, [1] * 3, np.zeros((3, 1, nq, D)))
        check(f"replay {i}", host(eager["out"]), ref, attention_bar("bf16", host(eager["q"]), k, ref, mag, D ** -0.5, n))


def test_another_stream_and_two_streams_at_once():
    c = Cache(16, "bf16", 1, 128, 64, [2000, 700])
    q = torch.randn(2, 3, 8, 128, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    kv = ints([2000, 700])
    want = px().paged_attention(q, c.px, kv)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(10):
        for s in (a, b):
            outs.append(px().paged_attention(q, c.px, kv, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_binding_refuses():
    c = Cache(17, "bf16", 2, 64, 16, [40, 40])
    q, kv = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device="cuda"), ints([40, 40])
    f = px().paged_attention
    for bad in (dict(out=q[:, :, :2]), dict(out=torch.zeros(2, 1, 4, 64, device="cuda")), dict(new_len=ints([1])),
                dict(workspace=torch.zeros(4))):
        with pytest.raises(ValueError):
            f(q, c.px, kv, **bad)
    for x in (q[:1], q[..., :32], q.cpu(), q[0]):
        with pytest.raises(ValueError):
            f(x, c.px, kv)
    with pytest.raises(ValueError):
        f(q, c.px, kv.long())
    with pytest.raises(px().PhyaiError):
        f(q[:, :, :3], c.px, kv)
    with pytest.raises(px().PhyaiError):
        f(q, c.px, kv, max_kv_len=c.px.capacity + 1)
    with pytest.raises(px().PhyaiError):
        f(q.float(), c.px, kv, out=None)
    for args in ((c.k, c.v[:-1], c.table), (c.k, c.v.float(), c.table), (c.k, c.v, c.table.long()),
                 (c.k, c.v, c.table, torch.ones(2, device="cuda"), torch.ones(2, device="cuda")),
                 (c.k.view(torch.uint8)[..., :64], c.v.view(torch.uint8)[..., :64], c.table)):
        with pytest.raises(ValueError):
            px().PagedCache(*args)
    assert f(q[:, :0], c.px, kv).shape == (2, 0, 4, 64)
