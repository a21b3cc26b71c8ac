"""Argument checks and sizes of the paged caches and rotary positions, and the frequencies of the scalings (nothing is launched, no
GPU needed)."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv

OK, BAD, NO = gkv.GKV_OK, gkv.GKV_ERR_INVALID_ARG, gkv.GKV_ERR_UNSUPPORTED
A = 1 << 20     # an aligned address that is never looked at
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


def pages(**over):
    kw = dict(format=gkv.GKV_STORE_INT8, n_q_heads=8, n_kv_heads=2, head_dim=128, n_pages=40, page_size=16, token_major=0, k=A, v=A, k_scale=A, v_scale=A)
    kw.update(over)
    return gkv.gkv_pages(**kw)


def table(**over):
    kw = dict(page=A, stride=10, batch=6, width=10)
    kw.update(over)
    return gkv.gkv_page_table(**kw)


def rotary(**over):
    kw = dict(head_dim=128, rot_dim=128, interleaved=0, factor=1.0, turns=A)
    kw.update(over)
    return gkv.gkv_rotary(**kw)


def ref(x):
    return None if x is None else ctypes.byref(x)


def copy(g, t, k=A, v=A, strides=(4096, 256, 128), first=None, count=None, n=4, rot=None, pos=None, ps=(0, 0), read=False):
    L = gkv.lib()
    if read:
        return L.gkv_pages_read(ref(g), ref(t), k, v, *strides, first, count, n, None)
    return L.gkv_pages_append(ref(g), ref(t), k, v, *strides, first, count, n, ref(rot), pos, *ps, None)


def attn(g, t, length=A, max_len=0, q=A, qs=1024, k_new=None, v_new=None, kvs=256, rot=None, pos=None, out=A, lse=None, ws=A, ws_bytes=1 << 40):
    return gkv.lib().gkv_pages_attn(ref(g), ref(t), length, max_len, q, qs, k_new, v_new, kvs, ref(rot), pos, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", [
    (dict(format=4), BAD), (dict(format=-1), BAD), (dict(n_q_heads=0), BAD), (dict(n_kv_heads=0), BAD), (dict(n_q_heads=9), BAD),
    (dict(n_pages=0), BAD), (dict(page_size=0), BAD), (dict(page_size=-16), BAD), (dict(head_dim=64), NO), (dict(head_dim=0), BAD),
    (dict(n_q_heads=18), NO), (dict(page_size=65537), NO), (dict(n_pages=1 << 26), NO), (dict(n_pages=2 ** 31 - 1, page_size=65536), NO),
])
def test_shapes_that_no_call_takes(over, status):
    g, L = pages(**over), gkv.lib()
    assert L.gkv_pages_query_sizes(ref(g), ref(gkv.gkv_store_sizes())) == status
    assert L.gkv_pages_attn_workspace(ref(g), 4, ref(ctypes.c_uint64())) == status
    assert copy(g, table()) == status and copy(g, table(), read=True) == status and attn(g, table()) == status


@pytest.mark.parametrize("over,status", [(dict(k=0), BAD), (dict(v=0), BAD), (dict(k=A + 8), BAD), (dict(v=A + 8), BAD), (dict(k_scale=0), BAD),
                                         (dict(v_scale=A + 4), BAD)])
def test_buffers_that_no_call_takes(over, status):
    g = pages(**over)
    assert copy(g, table()) == status and copy(g, table(), read=True) == status and attn(g, table()) == status


@pytest.mark.parametrize("over,status", [
    (dict(page=0), BAD), (dict(page=A + 2), BAD), (dict(stride=-1), BAD), (dict(batch=0), BAD), (dict(width=0), BAD), (dict(width=-3), BAD),
    (dict(batch=65536), NO), (dict(width=(1 << 20) + 1), NO),
])
def test_tables_that_no_call_takes(over, status):
    t = table(**over)
    assert copy(pages(), t) == status and copy(pages(), t, read=True) == status and attn(pages(), t) == status


ROTARIES = [(dict(turns=0), BAD), (dict(turns=A + 4), BAD), (dict(rot_dim=0), BAD), (dict(rot_dim=3), BAD), (dict(rot_dim=130), BAD), (dict(head_dim=127), BAD),
            (dict(head_dim=0, rot_dim=2), BAD), (dict(factor=math.inf), BAD), (dict(factor=math.nan), BAD)]


@pytest.mark.parametrize("over,status", ROTARIES + [(dict(head_dim=64, rot_dim=64), BAD)])
def test_rotaries_that_no_paged_call_takes(over, status):
    r = rotary(**over)
    assert copy(pages(), table(), rot=r) == status and attn(pages(), table(), rot=r) == status


def test_null_arguments():
    L = gkv.lib()
    assert copy(None, table()) == BAD and copy(pages(), None) == BAD and attn(None, table()) == BAD and attn(pages(), None) == BAD
    assert L.gkv_pages_query_sizes(None, ref(gkv.gkv_store_sizes())) == BAD and L.gkv_pages_query_sizes(ref(pages()), None) == BAD
    assert L.gkv_pages_attn_workspace(ref(pages()), 4, None) == BAD and L.gkv_pages_attn_workspace(None, 4, ref(ctypes.c_uint64())) == BAD
    assert L.gkv_pages_attn_workspace(ref(pages()), 0, ref(ctypes.c_uint64())) == BAD
    assert L.gkv_pages_attn_workspace(ref(pages()), 65536, ref(ctypes.c_uint64())) == NO


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(k=0), BAD), (dict(v=0), BAD), (dict(k=A + 2), BAD), (dict(v=A + 8), BAD), (dict(n=-1), BAD), (dict(strides=(4096, 256, 4)), BAD),
    (dict(strides=(4096, 252, 128)), BAD), (dict(strides=(-8, 256, 128)), BAD), (dict(first=A + 2), BAD), (dict(count=A + 1), BAD),
    (dict(n=1 << 29), NO), (dict(n=0), OK), (dict(n=0, k=0, v=0), OK),
])
def test_append_and_read_arguments(read, kw, status):
    assert copy(pages(), table(), read=read, **kw) == status


@pytest.mark.parametrize("kw,status", [(dict(pos=A + 2), BAD), (dict(pos=A, ps=(-1, 1)), BAD), (dict(pos=A, ps=(4, -1)), BAD)])
def test_positions_of_an_append(kw, status):
    assert copy(pages(), table(), rot=rotary(), **kw) == status


@pytest.mark.parametrize("n,strides", [(4, (0, 256, 128)), (4, (4096, 0, 128)), (4, (4096, 256, 0)), (4, (4096, 256, 120)), (4, (1016, 256, 128))])
def test_read_refuses_a_target_whose_rows_overlap(n, strides):
    assert copy(pages(), table(), v=2 * A, strides=strides, n=n, read=True) == BAD


def test_read_refuses_one_target_for_both():
    assert copy(pages(), table(), n=1, read=True) == BAD


@pytest.mark.parametrize("kw,status", [
    (dict(length=0), BAD), (dict(q=0), BAD), (dict(out=0), BAD), (dict(q=A + 8), BAD), (dict(out=A + 8), BAD), (dict(length=A + 2), BAD), (dict(lse=A + 2), BAD),
    (dict(qs=-8), BAD), (dict(qs=1020), BAD), (dict(k_new=A), BAD), (dict(v_new=A), BAD), (dict(k_new=A + 8, v_new=A), BAD), (dict(k_new=A, v_new=A + 8), BAD),
    (dict(k_new=A, v_new=A, kvs=100), BAD), (dict(k_new=A, v_new=A, kvs=-8), BAD), (dict(max_len=-1), BAD), (dict(max_len=161), BAD), (dict(ws=0), BAD),
    (dict(ws=A + 8), BAD), (dict(ws_bytes=1000), BAD), (dict(pos=A + 2), BAD),
])
def test_attention_arguments(kw, status):
    assert attn(pages(), table(), **kw) == status


def test_sizes():
    for fmt, row, scales in ((0, 256, 0), (1, 128, 1), (2, 128, 1), (3, 64, 4)):
        s = gkv.gkv_pages_query_sizes(pages(format=fmt, token_major=1))
        assert s.k == s.v == 40 * 16 * 2 * row and s.k_scale == s.v_scale == 40 * 16 * 2 * scales * 2


# ---------------------------------------------------------------------------------------------- rotation
def rows(**over):
    kw = dict(x=A, y=A, n_heads=3, x_stride=(3 * 4 * 128, 3 * 128, 128), y_stride=(3 * 4 * 128, 3 * 128, 128))
    kw.update(over)
    r = gkv.gkv_rotary_rows(kw["x"], kw["y"])
    r.n_heads = kw["n_heads"]
    for i in range(3):
        r.x_stride[i], r.y_stride[i] = kw["x_stride"][i], kw["y_stride"][i]
    return r


def apply(r=None, type=0, batch=2, n=4, pos=A, ps=(4, 1), count=None, q=None, k=None):
    return gkv.lib().gkv_rotary_apply(ref(r or rotary()), type, batch, n, pos, *ps, count, ref(q or rows()), ref(k), 0, None)


@pytest.mark.parametrize("over,status", ROTARIES + [(dict(head_dim=514, rot_dim=64), BAD)])
def test_rotaries_that_no_call_takes(over, status):
    assert apply(rotary(**over)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), BAD), (dict(type=-1), BAD), (dict(batch=0), BAD), (dict(batch=65536), NO), (dict(n=-1), BAD), (dict(n=0), OK), (dict(n=0, pos=0), OK),
    (dict(pos=0), BAD), (dict(pos=A + 2), BAD), (dict(ps=(-1, 1)), BAD), (dict(ps=(4, -1)), BAD), (dict(count=A + 2), BAD), (dict(q=rows(n_heads=0)), BAD),
    (dict(q=rows(x=0)), BAD), (dict(q=rows(y=0)), BAD), (dict(q=rows(x=A + 1, y=A + 1)), BAD), (dict(type=2, q=rows(x=A + 2, y=A + 2)), BAD),
    (dict(q=rows(x_stride=(1536, -384, 128), y_stride=(1536, -384, 128))), BAD),
    (dict(q=rows(x_stride=(1536, 384, 128), y_stride=(1536, 512, 128))), BAD),            # in place with different strides
    (dict(q=rows(y=2 * A, y_stride=(1536, 384, 64))), BAD), (dict(q=rows(y=2 * A, y_stride=(1536, 0, 128))), BAD),
    (dict(q=rows(y=2 * A, y_stride=(0, 384, 128))), BAD), (dict(q=rows(y=2 * A, y_stride=(1528, 384, 128))), BAD),
    (dict(k=rows(x=2 * A, y=A)), BAD),                                                        # one target for both
    (dict(q=rows(n_heads=1 << 29, x_stride=(1 << 40, 1 << 38, 128), y_stride=(1 << 40, 1 << 38, 128))), NO),
])
def test_rotation_arguments(kw, status):
    assert apply(**kw) == status


def test_rotation_null_arguments():
    L = gkv.lib()
    assert L.gkv_rotary_apply(None, 0, 2, 4, A, 4, 1, None, ref(rows()), None, 0, None) == BAD
    assert L.gkv_rotary_apply(ref(rotary()), 0, 2, 4, A, 4, 1, None, None, None, 0, None) == BAD


def test_turns_are_the_nearest_multiple():
    f = [1.0, 0.5, 1e-4, 3.7e-9, 0.0, 2 * math.pi, 7.0, 1e6, -0.3, 2.0 ** -70]
    got = gkv.gkv_rotary_turns(f)
    for x, t in zip(f, got):
        want = Fraction(x) / (2 * PI) * 2 ** 64
        off = (want - t) % 2 ** 64
        # 2^-1 by rounding, and |x / 2pi| 2^-64 2^64 for the quotient in 64 bits of mantissa (1 / 2pi is rounded, the division is)
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + 2 * abs(Fraction(x)) / (2 * PI) + 1, x
    with pytest.raises(gkv.GKVError):
        gkv.gkv_rotary_turns([math.inf])
    with pytest.raises(gkv.GKVError):
        gkv.gkv_rotary_turns([math.nan])
    with pytest.raises(gkv.GKVError):
        gkv.gkv_rotary_turns([2.0 ** 21])
    assert gkv.gkv_rotary_turns([]) == []


def close(got, want):
    assert len(got) == len(want)
    np.testing.assert_allclose(got, want, rtol=1e-13)      # a few roundings of 2^-53, pow's among them


@pytest.mark.parametrize("rot", [2, 32, 64, 128, 256])
def test_frequencies(rot):
    base = np.array([10000.0 ** (-2 * i / rot) for i in range(rot // 2)])
    plain, one = gkv.gkv_rotary_frequencies(1e4, rot)
    close(plain, base)
    assert one == 1
    close(gkv.gkv_rotary_frequencies(1e4, rot, gkv.GKV_ROTARY_LINEAR, 4)[0], base / 4)
    ntk = gkv.gkv_rotary_frequencies(1e4, rot, gkv.GKV_ROTARY_NTK, 4)[0]
    if rot > 2:        # the longest wave is stretched by the whole scale, the shortest not at all
        close([ntk[0], ntk[-1]], [base[0], base[-1] / 4])
    else:
        close(ntk, base)
    wave, one = gkv.gkv_rotary_frequencies(1e4, rot, gkv.GKV_ROTARY_WAVELENGTH, 8, 8192, 1, 4)
    assert one == 1
    for f, w in zip(base, wave):
        turns = 8192 * f / (2 * math.pi)
        s = min(max((turns - 1) / 3, 0), 1)
        close([w], [s * f + (1 - s) * f / 8])
    yarn, factor = gkv.gkv_rotary_frequencies(1e4, rot, gkv.GKV_ROTARY_YARN, 16, 4096, 1, 32)
    assert factor == np.float32(0.1 * math.log(16) + 1)
    d = lambda turns: rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(1e4))  # noqa: E731
    a, b = max(math.floor(d(32)), 0), min(math.ceil(d(1)), rot - 1)
    for i, (f, y) in enumerate(zip(base, yarn)):
        s = min(max((i - a) / max(b - a, 0.001), 0), 1)
        close([y], [f * (1 - s) + f / 16 * s])


@pytest.mark.parametrize("args", [(1.0, 64), (math.nan, 64), (math.inf, 64), (1e4, 63), (1e4, 0), (1e4, 514), (1e4, 64, 5), (1e4, 64, -1), (1e4, 64, 1, 0.5),
                                  (1e4, 64, 1, math.nan), (1e4, 64, 3, 8, 0, 1, 4), (1e4, 64, 3, 8, 4096, 0, 4), (1e4, 64, 4, 8, 4096, 4, 4),
                                  (1e4, 64, 4, 8, math.inf, 1, 4), (1e4, 64, 4, 8, 4096, 1, math.nan)])
def test_frequencies_that_are_refused(args):
    with pytest.raises(gkv.GKVError) as e:
        gkv.gkv_rotary_frequencies(*args)
    assert e.value.status == BAD
    assert gkv.lib().gkv_rotary_frequencies(1e4, 64, 0, 1, 0, 0, 0, None, None) == BAD


def test_holders_refuse():
    for kw in (dict(fmt="fp8"), dict(page_size=0), dict(pages=2 ** 31), dict(max_batch=0), dict(h_q=9), dict(device="cpu")):
        args = dict(fmt="int8", pages=4, page_size=16, h_q=8, h_kv=2, max_batch=2, device="cpu") | kw
        with pytest.raises((ValueError, gkv.GKVError)):
            gkv.PagedStore(args.pop("fmt"), **args)
    with pytest.raises(ValueError):
        gkv.PagedStore("bf16", pages=4, page_size=16, h_q=8, h_kv=2, max_batch=2, buffers=[torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)])
    with pytest.raises(ValueError):
        gkv.PagedStore("bf16", pages=4, page_size=16, h_q=8, h_kv=2, max_batch=2, token_major=True,
                       buffers=[torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)] * 2)
    for args, kw in (([[]], {}), ([[1.0] * 65], {}), ([[1.0]], dict(factor=math.inf)), ([[1.0]], dict(head_dim=514)), ([[1.0]], dict(head_dim=3)),
                     ([[1.0]], dict(device="cpu"))):
        with pytest.raises(ValueError):
            gkv.Rotary(*args, **(dict(device="cpu") | kw))
    with pytest.raises(ValueError):
        gkv.Rotary.scaled(1e4, scaling="cubic", device="cpu")
