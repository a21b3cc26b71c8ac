"""The key/value stores' argument checks and sizes (nothing is launched, no GPU needed), and pins of their fp64 reference."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
import store_reference as ref

OK, BAD, NO = gkv.GKV_OK, gkv.GKV_ERR_INVALID_ARG, gkv.GKV_ERR_UNSUPPORTED
A = 1 << 20     # an aligned address that is never looked at


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


def store(**over):
    kw = dict(format=gkv.GKV_STORE_INT8, batch=6, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=100, k=A, v=A, k_scale=A, v_scale=A)
    kw.update(over)
    return gkv.gkv_store(**kw)


SHAPES = [
    (dict(format=4), BAD), (dict(format=-1), BAD), (dict(batch=0), BAD), (dict(n_q_heads=0), BAD), (dict(n_kv_heads=0), BAD),
    (dict(capacity=0), BAD), (dict(capacity=-5), BAD), (dict(n_q_heads=9), BAD), (dict(head_dim=64), NO), (dict(n_q_heads=18), NO),
    (dict(batch=65536), NO), (dict(capacity=(1 << 24) + 1), NO),
]
POINTERS = [(dict(k=0), BAD), (dict(v=0), BAD), (dict(k=A + 8), BAD), (dict(v=A + 8), BAD), (dict(k_scale=0), BAD), (dict(v_scale=A + 4), BAD)]


def call_write(s, k=A, v=A, strides=(4096, 256, 128), first=None, count=None, n=4, read=False):
    f = gkv.lib().gkv_store_read if read else gkv.lib().gkv_store_write
    return f(ctypes.byref(s), k, v, *strides, first, count, n, None)


def make_prefix(n=2, rows=64, lens=(10, 64), k=A, v=A):
    arr = (ctypes.c_int32 * max(1, len(lens)))(*lens)
    return gkv.gkv_prefix(n, rows, arr, k, v)


def call_attn(s, length=A, max_len=0, q=A, k_new=None, v_new=None, prefix=None, out=A, lse=None, ws=A, ws_bytes=1 << 40):
    return gkv.lib().gkv_store_attn(ctypes.byref(s), length, max_len, q, k_new, v_new, None if prefix is None else ctypes.byref(prefix),
                                    out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", SHAPES)
def test_shapes_that_no_call_takes(over, status):
    s = store(**over)
    sizes, ws = gkv.gkv_store_sizes(), ctypes.c_uint64()
    L = gkv.lib()
    assert L.gkv_store_query_sizes(ctypes.byref(s), ctypes.byref(sizes)) == status
    assert L.gkv_store_attn_workspace(ctypes.byref(s), 0, 0, ctypes.byref(ws)) == status
    assert call_write(s) == status and call_write(s, read=True) == status and call_attn(s) == status


@pytest.mark.parametrize("over,status", POINTERS)
def test_buffers_that_no_call_takes(over, status):
    s = store(**over)
    assert call_write(s) == status and call_write(s, read=True) == status and call_attn(s) == status


def test_null_arguments():
    L, s = gkv.lib(), store()
    assert L.gkv_store_query_sizes(None, ctypes.byref(gkv.gkv_store_sizes())) == BAD
    assert L.gkv_store_query_sizes(ctypes.byref(s), None) == BAD
    assert L.gkv_store_attn_workspace(ctypes.byref(s), 0, 0, None) == BAD
    assert L.gkv_store_write(None, A, A, 8, 8, 8, None, None, 1, None) == BAD
    assert L.gkv_store_attn(None, A, 0, A, None, None, None, A, None, A, 1 << 40, None) == BAD
    assert L.gkv_decode_attn_prefix(None, 0, A, A, A, ctypes.byref(make_prefix()), A, A, 1 << 40, None) == BAD


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(k=0), BAD), (dict(v=0), BAD), (dict(k=A + 2), BAD), (dict(v=A + 8), BAD), (dict(n=-1), BAD),
    (dict(strides=(4096, 256, 4)), BAD), (dict(strides=(4096, 252, 128)), BAD), (dict(strides=(-8, 256, 128)), BAD),
    (dict(strides=(4100, 256, 128)), BAD), (dict(first=A + 2), BAD), (dict(count=A + 1), BAD), (dict(n=1 << 29), NO), (dict(n=0), OK),
])
def test_write_and_read_arguments(read, kw, status):
    assert call_write(store(), read=read, **kw) == status


@pytest.mark.parametrize("shape,n,strides", [
    (dict(), 4, (0, 256, 128)), (dict(), 4, (4096, 0, 128)), (dict(), 4, (4096, 256, 0)), (dict(), 4, (4096, 256, 120)),
    (dict(), 4, (4096, 248, 128)), (dict(), 4, (1016, 256, 128)), (dict(), 4, (256, 256, 128)), (dict(), 4, (2 ** 62, 2 ** 61, 128)),
    (dict(batch=1), 2, (0, 128, 128)), (dict(batch=1, n_kv_heads=1, n_q_heads=1), 2, (0, 0, 0)),
])
def test_read_refuses_a_target_whose_rows_overlap(shape, n, strides):
    assert call_write(store(**shape), v=2 * A, strides=strides, n=n, read=True) == BAD


def test_read_refuses_one_target_for_both():
    assert call_write(store(), n=1, read=True) == BAD


@pytest.mark.parametrize("kw,status", [
    (dict(length=0), BAD), (dict(q=0), BAD), (dict(out=0), BAD), (dict(q=A + 8), BAD), (dict(out=A + 8), BAD), (dict(length=A + 2), BAD),
    (dict(lse=A + 2), BAD), (dict(k_new=A), BAD), (dict(v_new=A), BAD), (dict(k_new=A + 8, v_new=A), BAD), (dict(k_new=A, v_new=A + 8), BAD),
    (dict(max_len=-1), BAD), (dict(max_len=101), BAD), (dict(ws=0), BAD), (dict(ws=A + 8), BAD), (dict(ws_bytes=1000), BAD),
    (dict(prefix=make_prefix(n=0)), BAD), (dict(prefix=make_prefix(n=65)), BAD), (dict(prefix=make_prefix(n=4, lens=(1, 1, 1, 1))), BAD),
    (dict(prefix=make_prefix(lens=(10, 65))), BAD), (dict(prefix=make_prefix(lens=(-1, 64))), BAD), (dict(prefix=make_prefix(k=0)), BAD),
    (dict(prefix=make_prefix(v=A + 8)), BAD), (dict(prefix=make_prefix(rows=-1, lens=(0, 0))), BAD),
    (dict(prefix=make_prefix(rows=1 << 29, lens=(1, 1))), NO),
])
def test_attention_arguments(kw, status):
    assert call_attn(store(), **kw) == status


def test_a_prefix_needs_its_workspace():
    s = store()
    assert call_attn(s, prefix=make_prefix(), ws_bytes=gkv.gkv_store_attn_workspace(s)) == BAD
    small, large = gkv.gkv_store_attn_workspace(s, 2, 64), gkv.gkv_store_attn_workspace(s, 3, 64)
    assert gkv.gkv_store_attn_workspace(s) < small <= large        # enough for up to so many prefixes
    with pytest.raises(gkv.GKVError):
        gkv.gkv_store_attn_workspace(s, 4, 64)                      # does not divide the batch
    with pytest.raises(gkv.GKVError):
        gkv.gkv_store_attn_workspace(s, 2, -1)


@pytest.mark.parametrize("fmt,row,scales", [("bf16", 256, 0), ("e4m3", 128, 1), ("int8", 128, 1), ("int4", 64, 4)])
def test_sizes(fmt, row, scales):
    z = gkv.gkv_store_query_sizes(store(format=gkv.STORE_FORMATS[fmt], batch=3, capacity=1 << 24))
    assert z.k == z.v == 3 * 2 * (1 << 24) * row and z.k_scale == z.v_scale == 3 * 2 * (1 << 24) * scales * 2


def test_holder_refuses_tensors_that_do_not_fit():
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)
    with pytest.raises(ValueError):
        gkv.KVStore("fp8", batch=1, h_q=4, h_kv=1, capacity=16)
    with pytest.raises(ValueError):     # a scale buffer is missing
        gkv.KVStore("int8", batch=1, h_q=4, h_kv=1, capacity=16, buffers=(t(1, 1, 16, 128, d=torch.int8),) * 2)
    with pytest.raises(ValueError):     # codes of another type
        gkv.KVStore("int4", batch=1, h_q=4, h_kv=1, capacity=16, buffers=(t(1, 1, 16, 64, d=torch.int8),) * 2 + (t(1, 1, 16, 4),) * 2)
    with pytest.raises(ValueError):     # a prefix on the host
        gkv.Prefix(t(1, 1, 16, 128), t(1, 1, 16, 128), [16])
    with pytest.raises(gkv.GKVError):
        gkv.KVStore("int8", batch=1, h_q=9, h_kv=1, capacity=16)


def test_the_torch_module_refuses_what_is_not_on_the_device():
    call, s = gkv._torch_binding(), store()
    at = ctypes.addressof(s)
    kv, q, n = torch.zeros((6, 3, 2, 128), dtype=torch.bfloat16), torch.zeros((6, 8, 128), dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int32)
    for bad in (lambda: call.copy(False, at, 0, kv, kv, None, None), lambda: call.copy(True, at, 0, "k", kv, None, None),
                lambda: call.attn(at, 0, n, 0, q, None, None, 0, q, None, A, 1 << 40)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call.copy(False, at), lambda: call.attn(at, 0), lambda: call.bind(1)):
        with pytest.raises(TypeError):
            bad()


# ------------------------------------------------------------------ the reference itself
def test_reference_codes_against_torch_and_by_hand():
    rng = np.random.RandomState(5)
    x = torch.from_numpy(rng.randn(50, 128) * np.exp2(rng.randint(-20, 20, (50, 1)))).to(torch.bfloat16)
    c, s = ref.encode(x.double().numpy(), "e4m3")
    t = (x.float() / torch.from_numpy(s).float()).to(torch.float8_e4m3fn)
    assert (t.view(torch.uint8).numpy() == ref.pack(c, "e4m3")).all() and np.abs(c).max() <= 448 and (np.abs(c).max(-1) >= 224).all()   # above 224, rounded
    row = np.zeros(128)
    row[:4] = [254.0, 3.0, -5.0, 1.0]                      # scale 2: 1.5 -> 2, -2.5 -> -2, 0.5 -> 0 (ties to even)
    c, s = ref.encode(row[None], "int8")
    assert s[0, 0] == 2.0 and c[0, :4].tolist() == [127, 2, -2, 0]
    c, s = ref.encode(np.zeros((1, 128)), "int4")
    assert (c == 0).all() and (s == 2.0 ** -126).all() and (ref.pack(c, "int4") == 0x88).all()
    row[:] = 0
    row[32 + 4 * 3 + 2] = 7.0                              # element 2 of word 4 * 3 + 1, a high byte's low nibble
    assert ref.pack(ref.encode(row[None], "int4")[0], "int4")[0, 2 * 13 + 1] == 0x8F
    assert np.isnan(ref.encode(np.array([[np.inf] + [1.0] * 127]), "int8")[1]).all()
    for fmt in ("e4m3", "int8", "int4"):                   # off by at most half a step
        y = rng.randn(20, 128)
        c, s = ref.encode(y, fmt)
        err = np.abs(ref.values(c, s, fmt) - y)
        lim = np.maximum(np.abs(y) * 2.0 ** -4, s * 2.0 ** -10) if fmt == "e4m3" else np.repeat(s, 128 // s.shape[-1], -1) / 2
        assert (err <= lim * (1 + 1e-12)).all()


def test_reference_attention_against_torch():
    rng = np.random.RandomState(6)
    q, k, v = rng.randn(3, 128), rng.randn(17, 128), rng.randn(17, 128)
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(t)[None] for t in (q, k, v)))[0].numpy()
    out, lse, _, _ = ref.attend(q, k[:5], v[:5], k[5:], v[5:])
    assert np.abs(out - want).max() < 1e-12
    assert np.abs(lse - np.log(np.exp(q @ k.T / np.sqrt(128)).sum(-1))).max() < 1e-12
    out, lse, _, _ = ref.attend(q, k[:0], v[:0])
    assert (out == 0).all() and (lse == -np.inf).all()
