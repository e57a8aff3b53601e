"""Calls of the paged cache that its documentation allows or refuses, on the GPU."""
import pytest

import workloads as wl
from test_gpu_prefill import plm_cfg
from test_gpu_prefill_paged import new_cache

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def px():
    import paper_2608_03682_amd as m
    return m


def test_prefill_refuses_a_workspace_that_is_not_plain_memory_of_the_device():
    cfg = plm_cfg(batch=1)
    case = wl.make_prefill_case(cfg, seed=39)
    lm = px().PrefixLM(cfg, case.weights)
    c = new_cache(cfg, 1, 2048, 16)
    emb = torch.from_numpy(case.embeds[:, :4]).cuda()
    need = px().paged_attention_workspace(c, cfg.n_q_heads, 4, 1004)
    assert need > 0
    before = c.k.view(torch.int16).clone()
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(need),
                torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            lm.prefill_paged(emb, c, [1000], workspace=bad)
    with pytest.raises(px().PhyaiError, match="workspace"):
        lm.prefill_paged(emb, c, [1000], workspace=torch.zeros(need - 16, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(c.k.view(torch.int16), before), "a refused call wrote to the cache"
    # one of the stated size serves the call, and nothing behind it is written
    c.k.zero_(), c.v.zero_()
    room = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    lm.prefill_paged(emb, c, [1000], workspace=room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 0x5a).all() and (room[:need] != 0x5a).any()
    lm.close()


def test_a_number_beyond_32_bits_is_refused_and_not_cut():
    """Not the layer, window, length or row count that is left of it."""
    big = 2 ** 32
    k = torch.zeros(2, 3, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    c = px().PagedCache(k, k.clone(), table)
    q, lens = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    x = torch.ones(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(layer=big), dict(layer=big + 1), dict(layer=-big), dict(window=big + 5), dict(window=1 - big),
                dict(max_kv_len=big + 16)):
        with pytest.raises(ValueError, match="32 bits"):
            px().paged_attention(q, c, lens, **bad)
    with pytest.raises(ValueError, match="32 bits"):
        px().paged_append(c, x, x, lens, layer=big)
    with pytest.raises(ValueError, match="32 bits"):
        px().paged_gather(c, lens, big + 4, out=torch.zeros(1, device="cuda"))
    far = q.expand(1, big + 1, 2, 64)
    for f in (lambda: px().paged_attention(far, c, lens, out=far), lambda: px().qk_norm_rope(far, q_out=far),
              lambda: px().paged_append(c, x.expand(1, big + 1, 1, 64), x.expand(1, big + 1, 1, 64), lens),
              lambda: px().PagedCache(k[0, :1].expand(big + 1, 16, 1, 64), k[0, :1].expand(big + 1, 16, 1, 64), table)):
        with pytest.raises(ValueError, match="32 bits"):
            f()
    torch.cuda.synchronize()
    assert (k == 0).all()
    # what the library refuses itself it still does
    for bad in (dict(layer=2), dict(layer=-1), dict(window=-1), dict(max_kv_len=33)):
        with pytest.raises(px().PhyaiError):
            px().paged_attention(q, c, lens, **bad)


@pytest.mark.parametrize("d_mlp", [512, 256])
def test_a_handle_holds_no_buffer_for_the_paged_path_alone(d_mlp):
    """512 requests of 816 rows: what a row has by phyai_prefill (residual stream, norm, queries,
    attention, MLP, cosines, keys and values), the projected rows of a chunk within the MLP's
    (384 values, so 128 more than an MLP of 256 has)."""
    cfg = plm_cfg(batch=512, prefix_cap=816, prefix_max=816, d_mlp=d_mlp)
    case = wl.make_prefill_case(cfg.replace(batch=1), seed=1)
    rows, d, qd, D, L = 512 * 816, cfg.d_model, 256, cfg.head_dim, cfg.n_layers
    assert (cfg.n_q_heads + 2 * cfg.n_kv_heads) * D == 384
    row = 4 * d + 2 * d + 2 * 2 * qd + 2 * max(d_mlp, 384) + 8 * D // 2
    cached = L * 2 * 512 * 832 * D * 2
    px().PrefixLM(cfg.replace(batch=1), case.weights).close()      # the context, the library's code
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.mem_get_info()[0]
    lm = px().PrefixLM(cfg, case.weights)
    used = before - torch.cuda.mem_get_info()[0]
    lm.close()
    print(f"[memory] {used / 2 ** 20:.0f} MiB, rows and cache {(rows * row + cached) / 2 ** 20:.0f} MiB", flush=True)
    # weights, lengths and the parts of split products: below 100 MB; the projected rows are 321 MB
    assert used < rows * row + cached + 100e6
