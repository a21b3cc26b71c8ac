"""A store that is dropped while a stream other than the one it was made on still works on it."""
import gc

import pytest
import torch

import paper_2512_00504_b200 as gkv
from test_gpu_store import DEV, gen, ints, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["attn", "write", "read"])
def test_memory_of_a_dropped_store_is_not_handed_out_while_a_stream_works_on_it(call):
    gkv.build_library()
    gkv.build_binding()
    B, H, C = 4, 4, 4608
    gc.collect()
    torch.cuda.empty_cache()
    st = gkv.KVStore("int8", batch=B, h_q=28, h_kv=H, capacity=C, device=DEV)
    x, q = randn(gen(1), 2, B, 64, H, 128), randn(gen(2), B, 28, 128)
    out, n = torch.empty_like(q), ints([64] * B)
    st.write(x[0], x[1])
    st.attn(n, q, out)
    torch.cuda.synchronize()
    names = ("k", "v", "k_scale", "v_scale") + (("workspace",) if call == "attn" else ())
    held = {name: (getattr(st, name).data_ptr(), getattr(st, name).numel() * getattr(st, name).element_size()) for name in names}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)          # about 0.2 s
        {"attn": lambda: st.attn(n, q, out), "write": lambda: st.write(x[0], x[1]), "read": lambda: st.read(x[0], x[1])}[call]()
    del st
    new = [torch.empty(size, dtype=torch.uint8, device=DEV) for _, size in held.values() for _ in range(2)]
    busy = not side.query()
    torch.cuda.synchronize()
    assert busy, "the stream was done before the check"
    for t in new:                               # nothing of the store's is in the new tensors
        for name, (at, size) in held.items():
            assert t.data_ptr() + t.numel() <= at or t.data_ptr() >= at + size, name


def test_memory_of_a_dropped_store_comes_back_once_the_stream_is_done():
    gc.collect()
    torch.cuda.empty_cache()
    st = gkv.KVStore("int8", batch=4, h_q=28, h_kv=4, capacity=4608, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        st.write(*randn(gen(3), 2, 4, 8, 4, 128))
    at, size = st.k.data_ptr(), st.k.numel()
    torch.cuda.synchronize()
    del st
    gc.collect()
    new = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(8)]
    assert any(t.data_ptr() == at for t in new)
