"""What the binding of the paged cache checks before the library is called, without a GPU:
tensors on the host stand in for those of a device, and the handle is NULL, which the
library refuses, so that a call that passes the checks ends there."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest

import paper_2608_03682_amd as px
from test_paged_cpu import cache

torch = pytest.importorskip("torch")


@pytest.fixture
def on_host(monkeypatch):
    monkeypatch.setattr(px, "_elsewhere", lambda t, stream: False)
    monkeypatch.setattr(px, "_here", lambda t: 0)
    monkeypatch.setattr(px, "_ptr", lambda t: None if t is None else t.data_ptr())


def prefix_lm(d=64):
    lm = object.__new__(px.PrefixLM)
    lm.cfg = SimpleNamespace(d_model=d, n_q_heads=8)
    lm._h = None
    lm.device = torch.device("cpu")
    return lm


def paged(batch=2, tokens=4096 * 64):
    c = cache(batch=batch, max_pages=tokens // 64, table_stride=tokens // 64)
    return SimpleNamespace(_c=c, _ref=ctypes.byref(c), batch=batch, capacity=tokens, k=torch.zeros(1))


def prefill(lm=None, embeds=None, c=None, past=(100000, 0), **kw):
    (lm or prefix_lm()).prefill_paged(torch.zeros(2, 4, 64) if embeds is None else embeds, c or paged(), past, **kw)


def passes(**kw):
    """The checks of the binding let the call through to the library, which finds no handle."""
    with pytest.raises(px.PhyaiError, match="NULL handle"):
        prefill(**kw)


def test_prefill_refuses_a_workspace_that_is_not_plain_memory_of_the_device(on_host):
    need = px.paged_attention_workspace(paged(), 8, 4, 100004)
    assert need > 16
    passes()
    passes(workspace=torch.zeros(need, dtype=torch.uint8))
    for bad in (torch.zeros(need, dtype=torch.uint8, device="meta"),           # another device
                torch.zeros(1, dtype=torch.uint8).expand(need),                # states more bytes than it has
                torch.zeros(2 * need, dtype=torch.uint8)[::2]):                # its neighbours' bytes between
        with pytest.raises(ValueError, match="workspace"):
            prefill(workspace=bad)


@pytest.mark.parametrize("heads,rows,longest", [(8 + 2 ** 32, 4, 64), (8, 4 + 2 ** 32, 64), (8, 4, 64 + 2 ** 32), (8, 4, 64 - 2 ** 32)])
def test_a_number_beyond_32_bits_is_refused_and_not_cut(heads, rows, longest):
    px.paged_attention_workspace(paged(), 8, 4, 64)
    with pytest.raises(ValueError, match="32 bits"):
        px.paged_attention_workspace(paged(), heads, rows, longest)


@pytest.mark.parametrize("past,new", [
    ([2 ** 32 + 3, 0], None), ([0, -2 ** 32], None), ([3, 0], [1 + 2 ** 32, 1]), ([0, 2 ** 63], None), ([0.5, 0], None),
    ([float("nan"), 0], None), ([0, 0], [1.5, 1]), ([[3, 0], [5, 0]], None), (7, None), ([0], None), ([0, 0], [1]), (["3", "0"], None)])
def test_lengths_of_a_chunk_are_refused_and_not_cut(on_host, past, new):
    """past_len and new_len are host values of any integer type, or whole numbers; what 32 bits
    cannot hold used to wrap to a length within the bounds."""
    with pytest.raises(ValueError, match="past_len|new_len"):
        prefill(past=past, new_len=new)


@pytest.mark.parametrize("past", [[3, 0], (3, 0), np.array([3, 0, 9], np.int64), np.array([3.0, 0.0]), torch.tensor([3, 0]),
                                  np.array([3, 0], np.uint8)])
def test_lengths_of_a_chunk_of_any_host_type(on_host, past):
    passes(past=past)
    passes(past=past, new_len=past)


def test_prefill_refuses_tensors_of_another_device_than_the_handles(on_host):
    """The weights and buffers of a handle lie on the device that was current when it was loaded."""
    lm = prefix_lm()
    passes(lm=lm)
    lm.device = torch.device("meta")
    with pytest.raises(ValueError, match="handle"):
        prefill(lm=lm)
