"""What a cache or a prefix refuses before anything is launched (no GPU needed)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2512_00504_b200 as gkv

CUDA = torch.device("cuda:0")


def cache(monkeypatch, h_kv):
    """A cache without its context, and the list of the calls that it makes."""
    c = gkv.GKVCache.__new__(gkv.GKVCache)
    c.cfg, c.ctx, c.device, c.k = gkv.make_config(n_layers=1, batch=2, h_q=8, h_kv=h_kv, b=96, buffer=32, w=8, s=32), None, CUDA, SimpleNamespace(device=CUDA)
    calls = []
    monkeypatch.setattr(gkv, "gkv_decode_attn_prefix", lambda *a: calls.append(a))
    return c, calls


@pytest.mark.parametrize("h_kv,device,fits", [(2, CUDA, True), (1, CUDA, False), (4, CUDA, False), (2, torch.device("cuda:1"), False)])
def test_a_cache_refuses_a_prefix_of_other_heads_or_another_device(monkeypatch, h_kv, device, fits):
    c, calls = cache(monkeypatch, 2)
    prefix = SimpleNamespace(h_kv=h_kv, k=SimpleNamespace(device=device))
    if fits:
        c.decode_attn_prefix(0, None, None, None, prefix, None, None)
    else:
        with pytest.raises(ValueError, match="KV heads"):
            c.decode_attn_prefix(0, None, None, None, prefix, None, None)
    assert len(calls) == fits
