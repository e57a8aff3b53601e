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
