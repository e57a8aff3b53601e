"""The prefix LM fed in chunks over a paged cache (phyai_prefill_paged) against the
oracle, on the bar of phyai_prefill's cache: the same GEMM operands are rounded at
the same places, and the attention's output is one more of them, as there."""
import numpy as np
import pytest

import oracle
import oracle.paged as op
import workloads as wl
from gpu_helpers import compare, small_cfg
from test_gpu_prefill import check_kv, kv_bar, plm_cfg

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def px():
    import paper_2608_03682_amd as m
    return m


def new_cache(cfg, batch, tokens, page, dtype=None, seed=1):
    """Pools full of NaN, pages in random order."""
    dt = dtype or (torch.float32 if cfg.weight_dtype == "f32" else torch.bfloat16)
    per = -(-tokens // page)
    n = batch * per + 3
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:batch * per]
    table = order.view(batch, per).int().cuda()
    pool = torch.full((cfg.n_layers, n, page, cfg.n_kv_heads, cfg.head_dim), float("nan")).to(dt)
    sc = [torch.full((cfg.n_kv_heads,), s, device="cuda") for s in (0.02, 0.03)] if dt == torch.float8_e4m3fn else [None] * 2
    return px().PagedCache(pool.cuda(), pool.cuda(), table, *sc)


def chunked(cfg, case, B, lens, parts, causal, page=16, cache=None, lm=None, prefix_cap=None):
    """Feeds every request's tokens in chunks; request b's chunk i has parts[b][i] tokens."""
    own = lm is None
    lm = lm or px().PrefixLM(cfg, case.weights, max_batch=B)
    c = cache or new_cache(cfg, B, max(lens), page)
    past = np.zeros(B, np.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for i, up_to in enumerate(causal):
        new = np.array([p[i] for p in parts], np.int32)
        rows = max(1, int(new.max()))
        emb = torch.full((B, rows, cfg.d_model), float("nan"))
        for b in range(B):
            emb[b, :new[b]] = torch.from_numpy(np.asarray(case.embeds[b, past[b]:past[b] + new[b]]))
        lm.prefill_paged(emb.cuda(), c, past, new, causal=up_to, status=status)
        past += new
    got = px().paged_gather(c, torch.tensor(lens, dtype=torch.int32, device="cuda"), prefix_cap or cfg.prefix_cap)
    torch.cuda.synchronize()
    assert status.item() == 0
    if own:
        lm.close()
    return got


CASES = [
    ("bf16_dh64", dict(), 16),
    ("bf16_dh256_mqa", dict(head_dim=256, n_q_heads=2, d_model=512, prefix_cap=130, prefix_min=70, prefix_max=130), 64),
    ("bf16_dh128_gqa", dict(head_dim=128, n_q_heads=4, n_kv_heads=2, n_layers=3), 32),
    ("bf16_no_rope", dict(rope=False), 16),
    ("fp8_weights", dict(weight_dtype="fp8", d_mlp=2048), 16),
    ("fp4_weights", dict(weight_dtype="fp4"), 16),
    ("f32", dict(weight_dtype="f32", kv_dtype="f32"), 16),
]


@pytest.mark.parametrize("name,kw,page", CASES)
def test_chunks_match_the_oracle(name, kw, page):
    cfg = plm_cfg(batch=3, **kw)
    print(f"[case] prefill_paged {name}", flush=True)
    case = wl.make_prefill_case(cfg, seed=41)
    cap = cfg.prefix_cap
    # images as one block, text causal, single tokens; ragged, with a request that skips a chunk
    parts = [[cap - 20, 17, 1, 2], [31, 0, 1, 5], [1, 20, 1, 0]]
    causal = [False, True, True, True]
    lens = [sum(p) for p in parts]
    got = chunked(cfg, case, 3, lens, parts, causal, page).double().cpu().numpy()
    for b in range(3):
        ref = op.prefill_chunks(cfg, case.weights, case.embeds[b, :lens[b]], parts[b], causal)
        full = np.zeros(got[:, :, b].shape)
        full[:, :, :lens[b]] = ref
        check_kv(f"prefill_paged {name} request {b}", cfg, got[:, :, b:b + 1], full[:, :, None], [lens[b]])


@pytest.mark.parametrize("rows", [100, 40])
def test_one_block_is_phyai_prefill(rows):
    """One chunk of whole prefixes without a causal mask against phyai_prefill itself: two
    roundings of the same values, each within the bar of the oracle."""
    cfg = plm_cfg(batch=3, prefix_cap=rows, prefix_min=rows // 2, prefix_max=rows)
    case = wl.make_prefill_case(cfg, seed=43)
    lens = [int(n) for n in case.prefix_len]
    lm = px().PrefixLM(cfg, case.weights)
    want = lm.prefill(torch.from_numpy(case.embeds).cuda(), case.prefix_len).view(torch.bfloat16)
    got = chunked(cfg, case, 3, lens, [[n] for n in lens], [False], lm=lm)
    again = chunked(cfg, case, 3, lens, [[n] for n in lens], [False], lm=lm)
    lm.close()
    assert torch.equal(got, again)
    a, b = got.double().cpu().numpy(), want.double().cpu().numpy()
    assert np.abs(a - b).max() <= 2 * kv_bar(cfg, b)


def test_an_8_bit_cache_holds_the_first_layer_to_half_a_step():
    cfg = plm_cfg(batch=2)
    case = wl.make_prefill_case(cfg, seed=45)
    c = new_cache(cfg, 2, 60, 16, torch.float8_e4m3fn)
    got = chunked(cfg, case, 2, [60, 50], [[40, 20], [40, 10]], [False, True], cache=c).double().cpu().numpy()
    assert np.isfinite(got).all()
    for b, n in enumerate((60, 50)):
        ref = op.prefill_chunks(cfg, case.weights, case.embeds[b, :n], [40, n - 40], [False, True])[0]
        s = np.array([0.02, 0.03])[:, None, None]
        # half a code step, the rows' own bar, the gather's rounding
        bar = np.maximum(np.abs(ref) * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -7) + kv_bar(cfg, ref) + 2.0 ** -8 * np.abs(ref)
        assert (np.abs(got[0, :, b, :n] - ref) <= bar).all()


def test_chunks_then_denoise_match_the_oracle_chain():
    """Chunked prefill, gather, action expert, as a policy runs them."""
    ecfg = small_cfg("pi0")
    pcfg = plm_cfg(n_layers=ecfg.n_layers, n_kv_heads=ecfg.n_kv_heads, head_dim=ecfg.head_dim, prefix_cap=ecfg.prefix_cap,
                   batch=ecfg.batch, d_model=512, n_q_heads=8, d_mlp=1024)
    pcase, ecase = wl.make_prefill_case(pcfg, seed=37), wl.make_case(ecfg, seed=37)
    lens = [int(n) for n in pcase.prefix_len]
    parts = [[n - 12, 11, 1] for n in lens]
    causal = [False, True, True]
    kv = chunked(pcfg, pcase, ecfg.batch, lens, parts, causal)
    ex = px().Expert(ecfg, ecase.weights)
    y = ex.denoise(kv, pcase.prefix_len, torch.from_numpy(ecase.noise).cuda(), ecase.timesteps,
                   torch.from_numpy(ecase.state).cuda())
    torch.cuda.synchronize()
    got = y.cpu().numpy().astype(np.float64)
    ref_kv = np.zeros(tuple(kv.shape))
    for b, n in enumerate(lens):
        ref_kv[:, :, b, :n] = op.prefill_chunks(pcfg, pcase.weights, pcase.embeds[b, :n], parts[b], causal)
    stored = wl.bf16_bits_from_f32(ref_kv.astype(np.float32))
    ref = oracle.denoise(ecfg, ecase.weights, stored, pcase.prefix_len, ecase.noise, ecase.timesteps, ecase.state)
    compare("prefill_paged -> gather -> denoise", got, ref, ecfg)
    ex.close()


def test_arguments_are_checked():
    cfg = plm_cfg(batch=2)
    case = wl.make_prefill_case(cfg, seed=39)
    lm = px().PrefixLM(cfg, case.weights)
    c = new_cache(cfg, 2, 64, 16)
    emb = torch.zeros((2, 5, cfg.d_model), device="cuda")
    before = c.k.view(torch.int16).clone()
    for kw in (dict(past_len=[60, 0]), dict(past_len=[-1, 0]), dict(past_len=[0, 0], new_len=[6, 1]),
               dict(past_len=[0, 0], new_len=[1, -1])):
        with pytest.raises(px().PhyaiError):
            lm.prefill_paged(emb, c, **kw)
    with pytest.raises(ValueError):
        lm.prefill_paged(emb[:1], c, [0])
    with pytest.raises(ValueError):
        lm.prefill_paged(emb, c, [0])
    with pytest.raises(px().PhyaiError):
        lm.prefill_paged(torch.zeros((2, cfg.prefix_cap + 1, cfg.d_model), device="cuda"), new_cache(cfg, 2, 300, 16), [0, 0])
    with pytest.raises(px().PhyaiError):
        lm.prefill_paged(emb, new_cache(cfg.replace(n_layers=3), 2, 64, 16), [0, 0])
    with pytest.raises(px().PhyaiError):
        lm.prefill_paged(emb, new_cache(cfg, 2, 64, 16, torch.float32), [0, 0])
    with pytest.raises(px().PhyaiError):
        lm.prefill_paged(torch.zeros((3, 5, cfg.d_model), device="cuda"), new_cache(cfg, 3, 64, 16), [0, 0, 0])
    torch.cuda.synchronize()
    assert torch.equal(c.k.view(torch.int16), before), "a refused call wrote to the cache"
    # a page out of range: that request's tokens are missing, the others' are right
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = new_cache(cfg, 2, 64, 16)
    lm.prefill_paged(emb, good, [0, 0])
    c.page_table[0, 0] = -3
    lm.prefill_paged(emb, c, [0, 0], status=status)
    torch.cuda.synchronize()
    assert status.item() == px().PAGED_BAD_PAGE
    p, r = int(c.page_table[1, 0]), int(good.page_table[1, 0])
    assert torch.equal(c.k[:, p, :5], good.k[:, r, :5]) and torch.equal(c.v[:, p, :5], good.v[:, r, :5])
    lm.close()


def test_gemma_size_in_two_chunks():
    """The 18-layer model over 816 tokens: one block against phyai_prefill (two roundings
    of the same values), and 768 image tokens, then 48 of text, with the image tokens'
    keys and values those of a prefix of 768."""
    cfg = wl.CONFIGS["plm_gemma_bf16_b1"]
    case = wl.make_prefill_case(cfg, seed=0)
    lm = px().PrefixLM(cfg, case.weights)
    emb = torch.from_numpy(case.embeds).cuda()
    want = lm.prefill(emb, [816]).view(torch.bfloat16).double()
    one = chunked(cfg, case, 1, [816], [[816]], [False], 64, lm=lm).double()
    two = chunked(cfg, case, 1, [816], [[768, 48]], [False, True], 64, lm=lm).double()
    short = lm.prefill(emb, [768]).view(torch.bfloat16).double()[:, :, :, :768]
    lm.close()
    for l in range(cfg.n_layers):
        w = want[l].cpu().numpy()
        bar = 2 * kv_bar(cfg.replace(n_layers=l + 1), w)
        print(f"[parity] layer {l}: one block {np.abs(one[l].cpu().numpy() - w).max():.3e}, bar {bar:.3e}", flush=True)
        assert np.abs(one[l].cpu().numpy() - w).max() <= bar
        s = short[l].cpu().numpy()
        assert np.abs(two[l, :, :, :768].cpu().numpy() - s).max() <= 2 * kv_bar(cfg.replace(n_layers=l + 1), s)
    assert torch.isfinite(two).all()
