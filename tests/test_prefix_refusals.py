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


class OnDevice:
    """Stands for a contiguous bf16 tensor on the device."""
    dtype, device = torch.bfloat16, CUDA

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 63])
def test_numbers_that_32_bits_do_not_hold(monkeypatch, n):
    """They are refused, and not taken for what is left of them in 32 bits."""
    gkv.build_library()
    with pytest.raises(ValueError, match="32 bits"):
        gkv.Prefix(OnDevice(2, 2, 64, 128), OnDevice(2, 2, 64, 128), [3, n])
    for name in ("batch", "h_q", "h_kv", "capacity", "n_prefix", "max_prefix"):
        with pytest.raises(ValueError, match="32 bits"):
            gkv.KVStore("int8", **{**dict(batch=1, h_q=8, h_kv=2, capacity=16, device="cpu"), name: n})
    c, _ = cache(monkeypatch, 2)
    c.C = 128
    for args in ((n, 10), (1, n)):
        with pytest.raises(ValueError, match="32 bits"):
            c.prefix_workspace(*args)


def test_lengths_of_a_prefix():
    assert list(gkv.Prefix(OnDevice(2, 2, 64, 128), OnDevice(2, 2, 64, 128), [3, torch.tensor(64)])._len) == [3, 64]
    with pytest.raises(ValueError, match="lengths"):
        gkv.Prefix(OnDevice(2, 2, 64, 128), OnDevice(2, 2, 64, 128), [3])


def test_self_test_of_the_wait_needs_a_context():
    gkv.build_library()
    assert gkv.lib().gkv_selftest_prefix_wait(None) == gkv.GKV_ERR_INVALID_ARG
