"""Key/value stores on the GPU against the fp64 reference: quantised write and read back (bit-exact), decode attention over a
store with the new row appended, shared prefixes, and the prefix in front of a context's compressed cache."""
import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
import store_reference as ref

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
FORMATS = ["bf16", "e4m3", "int8", "int4"]


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(torch.bfloat16)


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def raw(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def wide_rows(seed, n):
    """Rows that go wrong easily: all magnitudes bf16 has, ties, zeros, single large elements, values at the scales' borders."""
    rng = np.random.RandomState(seed)
    x = rng.randn(n, 128) * np.exp2(rng.randint(-133, 120, (n, 1)).astype(float))
    x[0] = 0
    x[1] = rng.randint(-254, 255, 128) / 2.0
    x[1, 0] = 127                                        # int8 scale 1: halves are ties
    x[2] = rng.randint(-14, 15, 128) / 2.0
    x[2, ::32] = 7                                       # int4 scale 1: ties
    x[3] = 448 * rng.choice([-1, 1, 0.5, 0.25], 128)
    x[4] = 450 * rng.choice([-1, 1, 0.5, 0.25], 128)     # just above 448 (bf16 450)
    x[5] = 2.0 ** -133 * rng.randint(-3, 4, 128)         # subnormals
    x[6] = rng.randn(128) * 1e-3
    x[6, 77] = 3e38
    x[7] = np.exp2(rng.randint(-30, 1, 128))
    x[8, 64:96] = 0                                      # a zero group among others
    x[9] = 17 * 2.0 ** -4 * rng.choice([1, 3, 5, 7], 128)
    x[9, 0] = 256                                        # e4m3: ties between neighbouring codes
    return torch.from_numpy(np.clip(x, -3.3e38, 3.3e38)).to(torch.bfloat16).to(DEV)


def expect_codes(x, fmt):
    """bytes [..., row], scales fp64 [..., groups] of rows x."""
    if fmt == "bf16":
        return raw(x).reshape(x.shape[:-1] + (256,)), np.zeros(x.shape[:-1] + (0,))
    c, s = ref.encode(f64(x), fmt)
    return ref.pack(c, fmt), s


def dequantised(store):
    """The store's rows as fp64, by the reference's reading of its bytes."""
    got = []
    for codes, scale in ((store.k, store.k_scale), (store.v, store.v_scale)):
        if store.fmt == "bf16":
            got.append(f64(codes))
        elif store.fmt == "int4":
            b = codes.cpu().numpy().astype(np.int64)
            c = np.zeros(b.shape[:-1] + (128,))
            for e in range(128):
                w, i = 4 * (e % 32 // 4) + e // 32, e % 4
                c[..., e] = ((b[..., 2 * w + i // 2] >> (4 * (i % 2))) & 15) - 8
            got.append(ref.values(c, f64(scale), "int4"))
        else:
            got.append(ref.values(f64(codes.float()), f64(scale), store.fmt))
    return got


# ---------------------------------------------------------------------------------------------- write, read
@pytest.mark.parametrize("fmt", FORMATS)
def test_codes_of_all_magnitudes(fmt):
    n = 480
    k, v = wide_rows(1, n), wide_rows(2, n)
    st = gkv.KVStore(fmt, batch=1, h_q=6, h_kv=3, capacity=n // 3, device=DEV)
    st.write(k.view(1, n // 3, 3, 128), v.view(1, n // 3, 3, 128))
    for x, codes, scale in ((k, st.k, st.k_scale), (v, st.v, st.v_scale)):
        want, s = expect_codes(x.view(n // 3, 3, 128).transpose(0, 1).contiguous(), fmt)
        assert (raw(codes[0]).reshape(want.shape) == want).all()
        if fmt != "bf16":
            assert (f64(scale[0]) == s).all()
    back = torch.empty((2, 1, n // 3, 3, 128), dtype=torch.bfloat16, device=DEV)
    st.read(back[0], back[1])
    if fmt == "bf16":
        assert torch.equal(back[0].view(n, 128), k) and torch.equal(back[1].view(n, 128), v)
    else:
        for x, got in ((k, back[0]), (v, back[1])):
            want = ref.round_bf16(ref.values(*ref.encode(f64(x), fmt), fmt))
            assert (f64(got).reshape(n, 128) == want).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_ragged_rows_from_a_strided_source(fmt):
    B, T, H, Hq, C = 5, 37, 2, 6, 64
    g = gen(3)
    qkv = randn(g, B, T, Hq + 2 * H, 128)
    k, v = qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    first, count = [0, 27, 60, 3, -2], [37, 37, 37, 0, 9]     # the last ones reach past both ends of the store
    st = gkv.KVStore(fmt, batch=B, h_q=Hq, h_kv=H, capacity=C, device=DEV)
    bufs = [t for t in (st.k, st.v, st.k_scale, st.v_scale) if t is not None]
    for t in bufs:
        t.view(torch.uint8).fill_(0x3A)
    st.write(k, v, first=ints(first), count=ints(count))
    written = np.zeros((B, C), bool)
    for b in range(B):
        for t in range(count[b]):
            r = first[b] + t
            if 0 <= r < C:
                written[b, r] = True
                for x, codes, scale in ((k, st.k, st.k_scale), (v, st.v, st.v_scale)):
                    want, s = expect_codes(x[b, t], fmt)
                    assert (raw(codes[b, :, r]).reshape(want.shape) == want).all(), (b, t)
                    if scale is not None:
                        assert (f64(scale[b, :, r]) == s).all()
    for t in bufs:                                             # everything else is as it was
        assert (raw(t).reshape(B, H, C, -1).transpose(0, 2, 1, 3)[~written] == 0x3A).all()
    wide = torch.full((2, B, T + 3, H + 1, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    out = wide[:, :, :T, :H]
    st.read(out[0], out[1], first=ints(first), count=ints(count))
    vals = dequantised(st)
    keep = np.ones((B, T + 3, H + 1), bool)
    for b in range(B):
        for t in range(count[b]):
            if 0 <= first[b] + t < C:
                keep[b, t, :H] = False
                for i in range(2):
                    assert (f64(out[i, b, t]) == ref.round_bf16(vals[i][b, :, first[b] + t])).all()
    assert (f64(wide)[:, keep] == 7.0).all()


@pytest.mark.parametrize("fmt", FORMATS[1:])
def test_what_is_not_finite_reads_back_as_nan(fmt):
    x = randn(gen(4), 1, 4, 1, 128)
    x[0, 0, 0, 40] = float("inf")
    x[0, 1, 0, 41] = float("nan")
    x[0, 2, 0, 42] = float("-inf")
    st = gkv.KVStore(fmt, batch=1, h_q=4, h_kv=1, capacity=4, device=DEV)
    st.write(x, x)
    out = torch.zeros((2, 1, 4, 1, 128), dtype=torch.bfloat16, device=DEV)
    st.read(out[0], out[1])
    bad = torch.isnan(out[0, 0, :, 0])
    group = slice(32, 64) if fmt == "int4" else slice(0, 128)
    assert bad[:3, group].all() and not bad[3].any() and int(bad.sum()) == 3 * (group.stop - group.start)
    if fmt == "int4":
        assert torch.equal(torch.isfinite(out[1, 0, :3, 0]).sum(-1).cpu(), torch.tensor([96, 96, 96]))


def test_no_tokens_and_one_token():
    st = gkv.KVStore("int8", batch=2, h_q=2, h_kv=2, capacity=3, device=DEV)
    st.k.fill_(5)
    st.write(torch.empty((2, 0, 2, 128), dtype=torch.bfloat16, device=DEV), torch.empty((2, 0, 2, 128), dtype=torch.bfloat16, device=DEV))
    assert (st.k == 5).all()
    x = randn(gen(5), 2, 1, 2, 128)
    st.write(x, x, first=ints([2, 0]))
    want, _ = expect_codes(x[:, 0], "int8")
    assert (raw(st.k[0, :, 2]) == want[0]).all() and (raw(st.k[1, :, 0]) == want[1]).all() and (st.k[0, :, :2] == 5).all()


# ---------------------------------------------------------------------------------------------- attention
def filled(fmt, B, Hq, H, C, lens, seed, **kw):
    """A store with lens[b] rows of every sequence written and all other bytes such that using them shows (NaN, or 0xFF)."""
    g = gen(seed)
    st = gkv.KVStore(fmt, batch=B, h_q=Hq, h_kv=H, capacity=C, device=DEV, **kw)
    for t in (st.k, st.v, st.k_scale, st.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0xFF)          # NaN as bf16 rows, as scales and as 8-bit floats
    n = max(max(lens), 1)
    k, v = randn(g, B, n, H, 128), randn(g, B, n, H, 128)
    k *= torch.exp2(torch.randint(-3, 3, (B, n, H, 1), generator=g, device=DEV).float()).to(torch.bfloat16)
    v *= torch.exp2(torch.randint(-12, 4, (B, n, H, 1), generator=g, device=DEV).float()).to(torch.bfloat16)
    st.write(k, v, count=ints([max(x, 0) for x in lens]))
    return st, g


def check(st, lens, q, out, lse, appended=False, prefix=None, seqs=None, skip=()):
    """out and lse against the reference on the rows the store holds now."""
    vals = dequantised(st)
    B, g = st.batch, st.h_q // st.h_kv
    o, l = f64(out), f64(lse)
    for b in (range(B) if seqs is None else seqs):
        if b in skip:
            continue
        n = lens[b] + int(appended)
        for h in range(st.h_kv):
            kp = vp = None
            if prefix is not None:
                i = b // (B // prefix[0].shape[0])
                kp, vp = f64(prefix[0][i, h, :prefix[2][i]]), f64(prefix[1][i, h, :prefix[2][i]])
            hs = slice(h * g, (h + 1) * g)
            want, wl, tol, ltol = ref.attend(f64(q[b, hs]), vals[0][b, h, :n], vals[1][b, h, :n], kp, vp,
                                             ref.U_BF16 if st.fmt == "bf16" else ref.U_F16)
            err = np.abs(o[b, hs] - want)
            assert (err <= tol).all(), (b, h, n, float((err / tol).max()))
            if np.isinf(wl).any():
                assert (l[b, hs] == wl).all()
            else:
                assert (np.abs(l[b, hs] - wl) <= ltol).all(), (b, h, n, float((np.abs(l[b, hs] - wl) / ltol).max()))


def attn_case(fmt, B, Hq, H, C, lens, seed, append, max_len=0, prefix=None, n_prefix=0, max_prefix=0, seqs=None):
    st, g = filled(fmt, B, Hq, H, C, lens, seed, n_prefix=n_prefix, max_prefix=max_prefix)
    q = randn(g, B, Hq, 128) * 1.5
    kn, vn = (randn(g, B, H, 128), randn(g, B, H, 128)) if append else (None, None)
    out = torch.full((B, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((B, Hq), 7.0, device=DEV)
    before = [raw(t).copy() for t in (st.k, st.v)]
    pre = None if prefix is None else gkv.Prefix(*prefix)
    st.attn(ints(lens), q, out, k_new=kn, v_new=vn, prefix=pre, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    after = [raw(t) for t in (st.k, st.v)]
    for x, y, new in zip(before, after, (kn, vn)):
        x, y = (t.reshape(B, H, C, -1) for t in (x, y))
        if append:
            want, _ = expect_codes(new, fmt)
            for b in range(B):
                if lens[b] >= 0:
                    assert (y[b, :, lens[b]] == want[b]).all()
                    x[b, :, lens[b]] = y[b, :, lens[b]]
        assert (x == y).all()                         # nothing but the new rows was written
    check(st, lens, q, out, lse, append, prefix, seqs, skip=[b for b in range(B) if lens[b] < 0])
    for b in range(B):
        if lens[b] < 0:
            assert (out[b] == 7).all() and (lse[b] == 7).all()
    return st


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_at_every_small_length(fmt, append):
    lens = list(range(0, 36)) + [47, 48, 49, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257]
    attn_case(fmt, len(lens), 14, 2, 260, lens, 11, append)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (6, 3), (4, 1), (5, 1), (28, 4), (16, 2)])
def test_attention_head_layouts(fmt, h_q, h_kv):
    attn_case(fmt, 3, h_q, h_kv, 300, [299, 5, 130], 12, True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,C,lens,max_len", [
    (1, 640, [639], 639), (1, 2000, [1999], 0), (2, 5000, [4999, 17], 4999), (3, 777, [776, 0, 400], 100),    # a max_len that is too small
    (2, 1024, [1024, 1000], 1024),
])
def test_attention_with_few_units_is_split(fmt, B, C, lens, max_len):
    attn_case(fmt, B, 8, 2, C, lens, 13, append=max(lens) < C, max_len=max_len)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_of_a_large_batch_with_sequences_left_out(fmt):
    rng = np.random.RandomState(14)
    B = 130
    lens = rng.randint(0, 150, B)
    lens[rng.choice(B, 30, replace=False)] = -1
    attn_case(fmt, B, 16, 4, 151, [int(x) for x in lens], 14, True, seqs=range(0, B, 3))


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("batch", [2, 300])     # split and whole units
def test_lengths_that_do_not_fit_give_nan_and_write_nothing(append, batch):
    C = 40
    lens = [10] * batch
    lens[0] = C + 1
    lens[1] = C if append else C + 7
    st, g = filled("int8", batch, 8, 2, C, [10] * batch, 15)
    q, kn = randn(g, batch, 8, 128), randn(g, batch, 2, 128)
    out, lse = torch.zeros((batch, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((batch, 8), device=DEV)
    before = raw(st.k)[0:2].copy()
    st.attn(ints(lens), q, out, k_new=kn if append else None, v_new=kn if append else None, lse=lse)
    assert torch.isnan(out[:2]).all() and torch.isnan(lse[:2]).all() and torch.isfinite(out[2:]).all()
    assert (raw(st.k)[0:2] == before).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_extreme_logits_and_scales(fmt):
    """Logits of +-10^4 (all weight on one key, later and earlier), V rows from 2^-100 to 2^100, zero rows."""
    B, H, n = 4, 1, 200
    st = gkv.KVStore(fmt, batch=B, h_q=3, h_kv=H, capacity=n, device=DEV)
    g = gen(16)
    k, v, q = randn(g, B, n, H, 128), randn(g, B, n, H, 128), randn(g, B, 3, 128)
    ramp = torch.linspace(-300, 300, n, device=DEV)
    k[0] = (q[0, 0] * ramp[:, None]).to(torch.bfloat16).view(n, 1, 128)
    k[1] = (q[1, 0] * ramp.flip(0)[:, None]).to(torch.bfloat16).view(n, 1, 128)
    v[2] = (v[2].float() * torch.exp2(torch.linspace(-100, 100, n, device=DEV))[:, None, None]).to(torch.bfloat16)
    v[3, ::2] = 0
    k[3, 1::3] = 0
    st.write(k, v)
    out, lse = torch.empty((B, 3, 128), dtype=torch.bfloat16, device=DEV), torch.empty((B, 3), device=DEV)
    st.attn(ints([n] * B), q, out, lse=lse)
    check(st, [n] * B, q, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_rows_show_in_the_output(fmt):
    st, g = filled(fmt, 3, 4, 1, 64, [50, 50, 50], 17)
    x = randn(g, 3, 1, 1, 128)
    y = x.clone()
    y[1] = float("nan")
    st.write(y, x, first=ints([20] * 3))              # K of sequence 1
    z = x.clone()
    z[2, :, :, 100] = float("inf")
    st.write(x, z, first=ints([20] * 3), count=ints([0, 0, 1]))
    out, lse = torch.empty((3, 4, 128), dtype=torch.bfloat16, device=DEV), torch.empty((3, 4), device=DEV)
    st.attn(ints([50] * 3), randn(g, 3, 4, 128), out, lse=lse)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all() and torch.isnan(lse[1]).all() and torch.isfinite(lse[2]).all()
    bad = ~torch.isfinite(out[2])
    group = slice(96, 128) if fmt == "int4" else slice(100, 101) if fmt == "bf16" else slice(0, 128)
    assert bad[:, group].all() and int(bad.sum()) == 4 * (group.stop - group.start)


def test_rows_beyond_4_gb():
    C = 1 << 23                                       # 3 heads x 2^23 rows x 256 bytes: 6 GB of K
    st = gkv.KVStore("bf16", batch=1, h_q=3, h_kv=3, capacity=C, device=DEV)
    g = gen(18)
    first = C - 40
    k, v = randn(g, 1, 30, 3, 128), randn(g, 1, 30, 3, 128)
    st.write(k, v, first=ints([first]))
    back = torch.zeros((2, 1, 30, 3, 128), dtype=torch.bfloat16, device=DEV)
    st.read(back[0], back[1], first=ints([first]))
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    assert torch.equal(st.k[0, 2, first:first + 30], k[0, :, 2])
    del st
    # attention: head 1 of a store whose second head starts beyond 2 GB and ends beyond 4
    C = 1 << 24
    st = gkv.KVStore("int8", batch=1, h_q=3, h_kv=3, capacity=C, device=DEV)
    st.k_scale.fill_(2.0 ** -7); st.v_scale.fill_(2.0 ** -7)
    st.k.zero_()
    st.v.fill_(64)
    st.v[0, 2, -1000:] = -64
    q = randn(g, 1, 3, 128)
    out, lse = torch.empty((1, 3, 128), dtype=torch.bfloat16, device=DEV), torch.empty((1, 3), device=DEV)
    st.attn(ints([C]), q, out, lse=lse)
    # all logits are 0: the mean of V, and log C; fp32 sums of 2^24 equal weights over many lanes are exact to 2^-12
    assert torch.allclose(lse, torch.full_like(lse, float(np.log(C))), rtol=2.0 ** -12, atol=0)
    assert torch.allclose(out.float(), torch.full((1, 3, 128), 0.5, device=DEV), rtol=2.0 ** -8 + 2000.0 / C, atol=0)


# ---------------------------------------------------------------------------------------------- shared prefixes
def prefix_rows(g, n, H, rows, lens):
    k, v = randn(g, n, H, rows, 128), randn(g, n, H, rows, 128)
    for i, m in enumerate(lens):                      # what lies behind a prefix must not matter
        k[i, :, m:] = float("nan")
        v[i, :, m:] = float("inf")
    return k, v, lens


@pytest.mark.parametrize("m", [0, 1, 2, 63, 127, 128, 129, 255, 256, 257, 400, 1000])
def test_prefix_lengths(m):
    g = gen(100 + m)
    attn_case("e4m3", 3, 14, 2, 40, [39, 0, 17], 21, False, prefix=prefix_rows(g, 1, 2, max(m, 1) + 3, [m]), n_prefix=1, max_prefix=m + 3)


@pytest.mark.parametrize("B,h_q,h_kv", [(1, 1, 1), (1, 8, 1), (15, 8, 1), (16, 8, 1), (17, 8, 1), (18, 7, 1), (19, 14, 2), (32, 16, 2),
                                        (33, 8, 1), (36, 7, 1), (37, 7, 1), (64, 8, 1), (130, 4, 1), (300, 1, 1)])
def test_prefix_row_blocks(B, h_q, h_kv):
    """Row counts around one tile (128), one block (256) and several blocks."""
    g = gen(200 + B)
    lens = [int(x) for x in np.random.RandomState(B).randint(0, 30, B)]
    attn_case("bf16", B, h_q, h_kv, 31, lens, 22, True, prefix=prefix_rows(g, 1, h_kv, 300, [291]), n_prefix=1, max_prefix=300,
              seqs=sorted({0, B // 3, B // 2, B - 1, 15 % B, 16 % B, 31 % B, 32 % B}))


@pytest.mark.parametrize("fmt", FORMATS)
def test_several_prefixes_of_different_lengths(fmt):
    g = gen(23)
    lens = [int(x) for x in np.random.RandomState(23).randint(-1, 90, 4 * 9)]
    attn_case(fmt, 36, 12, 3, 91, lens, 23, True, prefix=prefix_rows(g, 4, 3, 700, [700, 0, 129, 512]), n_prefix=4, max_prefix=700)


def test_only_a_prefix_and_nothing_at_all():
    g = gen(24)
    attn_case("int4", 6, 4, 1, 16, [0] * 6, 24, False, prefix=prefix_rows(g, 2, 1, 200, [0, 200]), n_prefix=2, max_prefix=200)
    attn_case("int8", 2, 4, 1, 16, [0, 0], 25, False, prefix=prefix_rows(g, 2, 1, 1, [0, 0]), n_prefix=2, max_prefix=1)


def test_a_long_prefix_with_logits_that_keep_rising():
    """Every key tile raises the running maximum (accumulators are rescaled each time), or none does."""
    for two_tiles, sign in ((False, 1), (True, 1), (True, -1)):
        B = 36 if two_tiles else 4
        g = gen(26)
        q = randn(g, B, 7, 128)
        m = 1500
        k, v = randn(g, 1, 1, m, 128), randn(g, 1, 1, m, 128)
        u = q.float().mean((0, 1)) + 0.3
        k += (sign * u[None, :] * torch.linspace(-60, 60, m, device=DEV)[:, None]).to(torch.bfloat16)
        st, _ = filled("bf16", B, 7, 1, 20, [9] * B, 27, n_prefix=1, max_prefix=m)
        out, lse = torch.empty((B, 7, 128), dtype=torch.bfloat16, device=DEV), torch.empty((B, 7), device=DEV)
        st.attn(ints([9] * B), q, out, lse=lse, prefix=gkv.Prefix(k, v, [m]))
        check(st, [9] * B, q, out, lse, prefix=(k, v, [m]), seqs=[0, 1, B - 1])


def test_nan_in_a_prefix_and_in_one_query():
    g = gen(28)
    k, v, lens = prefix_rows(g, 1, 1, 300, [300])
    st, _ = filled("e4m3", 5, 4, 1, 20, [9] * 5, 28, n_prefix=1, max_prefix=300)
    q = randn(g, 5, 4, 128)
    q[3, 2, 5] = float("nan")
    out = torch.empty((5, 4, 128), dtype=torch.bfloat16, device=DEV)
    st.attn(ints([9] * 5), q, out, prefix=gkv.Prefix(k, v, lens))
    bad = torch.isnan(out).all(-1)
    assert bad[3, 2] and int(bad.sum()) == 1 and int(torch.isnan(out).any(-1).sum()) == 1
    v[0, 0, 77, 64] = float("nan")
    st.attn(ints([9] * 5), q, out, prefix=gkv.Prefix(k, v, lens))
    assert torch.isnan(out[:, :, 64]).all() and torch.isfinite(out[0, :, :64]).all()
    v[0, 0, 77, 64] = 0
    k[0, 0, 200, 3] = float("nan")                    # a key: every row that sees it
    lse = torch.zeros((5, 4), device=DEV)
    st.attn(ints([9] * 5), q, out, prefix=gkv.Prefix(k, v, lens), lse=lse)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


# ---------------------------------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("fmt", ["e4m3", "int4"])
def test_prompt_write_then_decode_in_a_replayed_graph(fmt):
    """A prompt is quantised into the store, then tokens are decoded by replaying one captured step whose lengths grow on the
    device, on a stream of its own; the store is read back at the end."""
    B, Hq, H, C, T, steps, m = 3, 8, 2, 96, 61, 30, 140
    g = gen(31)
    k, v, lens = prefix_rows(g, 1, H, m, [m])
    prefix = gkv.Prefix(k, v, lens)
    st = gkv.KVStore(fmt, batch=B, h_q=Hq, h_kv=H, capacity=C, device=DEV, n_prefix=1, max_prefix=m)
    counts = [61, 40, 1]
    kp, vp = randn(g, B, T, H, 128), randn(g, B, T, H, 128)
    length = ints(counts)
    q, kn, vn = randn(g, B, Hq, 128), randn(g, B, H, 128), randn(g, B, H, 128)
    out, lse = torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((B, Hq), device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        st.write(kp, vp, count=length)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            st.attn(length, q, out, k_new=kn, v_new=vn, prefix=prefix, lse=lse, max_len=C - 1)
            length += 1
        for t in range(steps):
            q.copy_(randn(g, B, Hq, 128)); kn.copy_(randn(g, B, H, 128)); vn.copy_(randn(g, B, H, 128))
            graph.replay()
            if t % 7 == 0 or t == steps - 1:
                s.synchronize()
                check(st, [c + t for c in counts], q, out, lse, True, (k, v, lens))
        n = [c + steps for c in counts]
        back = torch.zeros((2, B, C, H, 128), dtype=torch.bfloat16, device=DEV)
        st.read(back[0], back[1], count=length)
    s.synchronize()
    assert length.tolist() == n
    for i, val in enumerate(dequantised(st)):
        for b in range(B):
            assert (f64(back[i, b, :n[b]]) == ref.round_bf16(val[b, :, :n[b]].transpose(1, 0, 2))).all()


def test_results_repeat_bit_for_bit_and_do_not_depend_on_the_workspace():
    g = gen(32)
    k, v, lens = prefix_rows(g, 1, 2, 600, [555])
    st, _ = filled("int8", 9, 14, 2, 700, [600 + i for i in range(9)], 33, n_prefix=1, max_prefix=600)
    q = randn(g, 9, 14, 128)
    length = ints([600 + i for i in range(9)])
    got = []
    for fill in (0, 0xFF, 0x7F):
        st.workspace.fill_(fill)
        out = torch.empty((9, 14, 128), dtype=torch.bfloat16, device=DEV)
        st.attn(length, q, out, prefix=gkv.Prefix(k, v, lens))
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_context_with_a_prefix_decodes_and_evicts():
    """gkv_decode_attn_prefix over a compressed cache: lengths advance, compressions are scored from window queries, and every
    step's output is attention over prefix and cache as they stand."""
    L, B, Hq, H, b, s, w = 2, 3, 8, 2, 48, 16, 16
    cfg = gkv.make_config(n_layers=L, batch=B, h_q=Hq, h_kv=H, b=b, buffer=24, w=w, s=s, fuse_window_scores=False)
    cache = gkv.GKVCache(cfg, DEV)
    g = gen(41)
    m = 333
    kp, vp, lens = prefix_rows(g, 1, H, m, [m])
    prefix, ws = gkv.Prefix(kp, vp, lens), cache.prefix_workspace(1, m)
    qs = [[] for _ in range(L)]
    n = 0
    for t in range(b + 3 * s):
        for layer in range(L):
            q, kn, vn = randn(g, B, Hq, 128), randn(g, B, H, 128), randn(g, B, H, 128)
            out = torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=DEV)
            cache.decode_attn_prefix(layer, q, kn, vn, prefix, out, ws)
            qs[layer].append(q)
            if t % 9 == 0 or t > b:
                view = gkv.KVStore("bf16", batch=B, h_q=Hq, h_kv=H, capacity=cache.C, buffers=(cache.k[layer], cache.v[layer]))
                lse = torch.full((B, Hq), 0.0, device=DEV)
                again = torch.empty_like(out)
                view2 = gkv.KVStore("bf16", batch=B, h_q=Hq, h_kv=H, capacity=cache.C, buffers=(cache.k[layer], cache.v[layer]),
                                    n_prefix=1, max_prefix=m)
                view2.attn(cache.len[0, layer], q, again, prefix=prefix, lse=lse)   # the row is in the cache now
                check(view, [n + 1] * B, q, out, lse, False, (kp, vp, lens), seqs=[t % B])
        n += 1
        assert cache.state(0)[0] == n and cache.len[0].unique().tolist() == [n]
        if (t + 1) % s == 0:
            for layer in range(L):
                cache.evict(layer, torch.stack(qs[layer][-w:], 2).contiguous())
            n = min(n, b)
            assert cache.state(L - 1)[0] == n and cache.len[0].unique().tolist() == [n]
    cache.poll()
    with pytest.raises(gkv.GKVError) as e:            # the ordinary calls still work on it, and a full cache is refused
        for _ in range(40):
            cache.decode_attn_prefix(0, q, kn, vn, prefix, out, ws)
    assert e.value.status == gkv.GKV_ERR_CAPACITY and cache.state(0)[0] == cache.C
    fused = gkv.GKVCache(gkv.make_config(n_layers=1, batch=B, h_q=Hq, h_kv=H, b=b, buffer=24, w=w, s=s), DEV)
    with pytest.raises(gkv.GKVError) as e:
        fused.decode_attn_prefix(0, q, kn, vn, prefix, out, fused.prefix_workspace(1, m))
    assert e.value.status == gkv.GKV_ERR_STATE


@pytest.mark.parametrize("seed", range(24))
def test_shapes_drawn_at_random(seed):
    rng = np.random.RandomState(900 + seed)
    fmt = FORMATS[seed % 4]
    h_kv = int(rng.choice([1, 2, 3, 8]))
    g_heads = int(rng.randint(1, 9))
    n_prefix = int(rng.choice([0, 1, 1, 2, 5]))
    B = max(1, n_prefix) * int(2 ** rng.uniform(0, 6.5 if n_prefix < 2 else 4))
    C = int(2 ** rng.uniform(2, 11))
    append = bool(rng.randint(2))
    lens = [int(x) for x in rng.randint(-1, C + (0 if append else 1), B)]
    prefix, rows = None, int(2 ** rng.uniform(0, 11))
    if n_prefix:
        plens = [int(x) for x in rng.randint(0, rows + 1, n_prefix)]
        prefix = prefix_rows(gen(950 + seed), n_prefix, h_kv, rows, plens)
    seqs = sorted(set(int(x) for x in rng.randint(0, B, 6)) | {0, B - 1})
    attn_case(fmt, B, h_kv * g_heads, h_kv, C, lens, 990 + seed, append, max_len=int(rng.choice([0, C, max(1, C // 3)])), prefix=prefix,
              n_prefix=n_prefix, max_prefix=rows, seqs=seqs)


def test_two_stores_on_two_streams_at_once():
    """Stores with workspaces of their own share nothing: what they give together is what each gives alone."""
    g = gen(51)
    k, v, lens = prefix_rows(g, 1, 2, 3000, [2900])
    prefix = gkv.Prefix(k, v, lens)
    cases = []
    for i, fmt in enumerate(("int4", "e4m3")):
        st, _ = filled(fmt, 24, 16, 2, 2000, [1990] * 24, 60 + i, n_prefix=1, max_prefix=3000)
        cases.append((st, randn(g, 24, 16, 128), torch.empty((24, 16, 128), dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()))
    length = ints([1990] * 24)
    alone = []
    for st, q, out, _ in cases:
        st.attn(length, q, out, prefix=prefix)
        alone.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for st, q, out, s in cases:
            with torch.cuda.stream(s):
                st.attn(length, q, out, prefix=prefix)
    torch.cuda.synchronize()
    for (_, _, out, _), want in zip(cases, alone):
        assert torch.equal(out, want)


def test_two_captured_graphs_share_a_workspace():
    g = gen(52)
    k, v, lens = prefix_rows(g, 1, 1, 700, [700])
    st, _ = filled("int8", 6, 8, 1, 900, [800] * 6, 53, n_prefix=1, max_prefix=700)
    q = randn(g, 6, 8, 128)
    short, long = ints([7, 0, 100, 3, 50, 1]), ints([800] * 6)
    outs = [torch.empty((6, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    calls = [lambda: st.attn(short, q, outs[0], prefix=gkv.Prefix(k, v, lens)), lambda: st.attn(long, q, outs[1], max_len=800)]
    want, graphs = [], []
    for call, out in zip(calls, outs):
        call()
        want.append(out.clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1, 0)):
        for out in outs:
            out.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_calls_refuse_tensors_that_do_not_fit():
    st = gkv.KVStore("int8", batch=2, h_q=8, h_kv=2, capacity=16, device=DEV)
    x = torch.zeros((2, 3, 2, 128), dtype=torch.bfloat16, device=DEV)
    q, out, length = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), ints([3, 3])
    bad_copies = [
        lambda: st.write(x.float(), x.float()), lambda: st.write(x[:1], x[:1]), lambda: st.write(x, x[:, :2]), lambda: st.write(x.cpu(), x.cpu()),
        lambda: st.write(x, x.permute(0, 1, 3, 2).contiguous().permute(0, 1, 3, 2)),                        # elements not next to each other
        lambda: st.write(x, torch.zeros((2, 2, 3, 128), dtype=torch.bfloat16, device=DEV).transpose(1, 2)),   # strides that differ
        lambda: st.read(x, x, first=ints([0])), lambda: st.read(x, x, count=torch.zeros(2, device=DEV)), lambda: st.write(None, x),
    ]
    kn = torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV)
    bad_attn = [
        lambda: st.attn(length.long(), q, out), lambda: st.attn(length.cpu(), q, out), lambda: st.attn(length, q[:, :4], out),
        lambda: st.attn(length, q.transpose(0, 1).contiguous().transpose(0, 1), out), lambda: st.attn(length, q, out.float()),
        lambda: st.attn(length, q, out, k_new=kn[:, :1], v_new=kn), lambda: st.attn(length, q, out, lse=torch.zeros((2, 4), device=DEV)),
        lambda: st.attn(length, q, out, prefix=gkv.Prefix(torch.zeros((1, 3, 8, 128), dtype=torch.bfloat16, device=DEV),
                                                          torch.zeros((1, 3, 8, 128), dtype=torch.bfloat16, device=DEV), [8])),   # heads
    ]
    for call in bad_copies + bad_attn:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: st.attn(length, q, out, k_new=kn), lambda: st.attn(length, q, out, max_len=17), lambda: st.attn(length, q, out, max_len=-1),
                 lambda: st.write(torch.zeros((2, 3, 2, 132), dtype=torch.bfloat16, device=DEV)[..., :128], torch.zeros((2, 3, 2, 132), dtype=torch.bfloat16, device=DEV)[..., :128]),
                 lambda: st.attn(length, q, out, prefix=gkv.Prefix(torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16, device=DEV),
                                                                   torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16, device=DEV), [8]))):   # no workspace for it
        with pytest.raises(gkv.GKVError) as e:
            call()
        assert e.value.status == gkv.GKV_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 0).all()


def masked_keys(g, q, n, H, spans):
    """K, V [B][n][H][128] where the keys of a sequence's span have a logit of -infinity (q is made positive in element 0)."""
    q[..., 0] = q[..., 0].abs() + 0.5
    k, v = randn(g, len(spans), n, H, 128), randn(g, len(spans), n, H, 128)
    for i, (a, b) in enumerate(spans):
        k[i, a:b, :, 0] = float("-inf")
    return k, v


def check_masked(q, out, lse, own, prefix):
    """own, prefix: per sequence K, V [n][H][128], span (or None). A key of weight 0 is a key that is not there."""
    g = q.shape[1] // own[0][0].shape[1]
    for b, (k, v, (x, y)) in enumerate(own):
        for h in range(k.shape[1]):
            keep = [i for i in range(len(k)) if not x <= i < y]
            kp = vp = None
            if prefix is not None:
                pk, pv, (s, e) = prefix[b]
                there = [i for i in range(len(pk)) if not s <= i < e]
                kp, vp = f64(pk[there, h]), f64(pv[there, h])
            hs = slice(h * g, (h + 1) * g)
            want, wl, tol, ltol = ref.attend(f64(q[b, hs]), f64(k[keep, h]), f64(v[keep, h]), kp, vp, ref.U_BF16)
            assert (np.abs(f64(out[b, hs]) - want) <= tol).all(), (b, h)
            if np.isinf(wl).any():
                assert (f64(lse[b, hs]) == wl).all()
            else:
                assert (np.abs(f64(lse[b, hs]) - wl) <= ltol).all(), (b, h)


@pytest.mark.parametrize("batch", [5, 200])      # units cut into pieces and whole ones
def test_own_keys_with_a_logit_of_minus_infinity(batch):
    n, H = 200, 2
    g = gen(61)
    q = randn(g, batch, 8, 128)
    spans = [(0, 100), (30, 150), (100, 200), (0, 200), (0, 199)] + [(0, 0)] * (batch - 5)
    k, v = masked_keys(g, q, n, H, spans)
    st = gkv.KVStore("bf16", batch=batch, h_q=8, h_kv=H, capacity=n, device=DEV)
    st.write(k, v)
    out, lse = torch.empty((batch, 8, 128), dtype=torch.bfloat16, device=DEV), torch.empty((batch, 8), device=DEV)
    st.attn(ints([n] * batch), q, out, lse=lse)
    check_masked(q[:5], out[:5], lse[:5], [(k[i], v[i], spans[i]) for i in range(5)], None)


@pytest.mark.parametrize("seqs", [3, 16, 32])    # rows of a tile that do not exist; the streams of an item share their rows; or not
@pytest.mark.parametrize("m,H,span", [(700, 1, (0, 130)), (700, 1, (0, 300)), (700, 1, (0, 699)), (700, 1, (0, 700)), (700, 1, (200, 500)),
                                      (5000, 16, (0, 700)), (5000, 16, (600, 3333)), (5000, 16, (0, 4999))])   # runs of several tiles
def test_prefix_keys_with_a_logit_of_minus_infinity(seqs, m, H, span):
    g = gen(62)
    q = randn(g, seqs, 8 * H, 128)
    pk, pv = masked_keys(g, q, m, H, [span])
    own = randn(g, 2, seqs, 3, H, 128)
    st = gkv.KVStore("bf16", batch=seqs, h_q=8 * H, h_kv=H, capacity=3, device=DEV, n_prefix=1, max_prefix=m)
    st.write(own[0], own[1])
    some = [0, seqs - 1]
    for n in (3, 0):                             # with rows of their own and without
        out, lse = torch.empty((seqs, 8 * H, 128), dtype=torch.bfloat16, device=DEV), torch.empty((seqs, 8 * H), device=DEV)
        prefix = gkv.Prefix(pk.transpose(1, 2).contiguous(), pv.transpose(1, 2).contiguous(), [m])
        st.attn(ints([n] * seqs), q, out, prefix=prefix, lse=lse)
        check_masked(q[some], out[some], lse[some], [(own[0, i, :n], own[1, i, :n], (0, 0)) for i in some], [(pk[0], pv[0], span)] * 2)


@pytest.mark.parametrize("where", ["own", "prefix"])
@pytest.mark.parametrize("seqs", [16, 32])
def test_values_near_the_end_of_the_range_under_rising_logits(where, seqs):
    """V of 2^90 and logits that go from -18 to 18 (52 in log2 units) and back every other tile of 128: outputs are finite, so all
    sums have to be."""
    m, H = (5000, 16) if where == "prefix" else (700, 1)
    g = gen(63)
    q = randn(g, 1, 1, 128).expand(seqs, 8 * H, 128).contiguous()
    unit = q[0, 0].float() / q[0, 0].float().square().sum() * 128 ** 0.5
    k = (unit * (torch.arange(m, device=DEV) // 256 % 2 * 36 - 18)[:, None]).to(torch.bfloat16).view(1, m, 1, 128).expand(1, m, H, 128)
    v = (randn(g, 1, m, H, 128).float() * 2.0 ** 90).to(torch.bfloat16)
    out, lse = torch.empty((seqs, 8 * H, 128), dtype=torch.bfloat16, device=DEV), torch.empty((seqs, 8 * H), device=DEV)
    st = gkv.KVStore("bf16", batch=seqs, h_q=8 * H, h_kv=H, capacity=m, device=DEV, n_prefix=1, max_prefix=m)
    if where == "own":
        seqs, out, lse = 16 * seqs, out.repeat(16, 1, 1), lse.repeat(16, 1)      # units whole
        q = q.repeat(16, 1, 1)
        st = gkv.KVStore("bf16", batch=seqs, h_q=8, h_kv=1, capacity=m, device=DEV)
        k, v = (t.expand(seqs, m, H, 128).contiguous() for t in (k, v))
        st.write(k, v)
        st.attn(ints([m] * seqs), q, out, lse=lse)
        check(st, [m] * seqs, q, out, lse, seqs=[0, seqs - 1])
    else:
        prefix = (k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous(), [m])
        st.attn(ints([0] * seqs), q, out, prefix=gkv.Prefix(*prefix), lse=lse)
        check(st, [0] * seqs, q, out, lse, prefix=prefix, seqs=[0])
    assert torch.isfinite(out).all()


def test_as_many_prefixes_as_there_may_be():
    B, H, rows = 128, 1, 140
    g = gen(64)
    lens = [(37 * i) % (rows + 1) for i in range(64)]
    prefix = prefix_rows(g, 64, H, rows, lens)
    attn_case("e4m3", B, 4, H, 9, [i % 9 for i in range(B)], 65, True, prefix=prefix, n_prefix=64, max_prefix=rows)


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_the_largest_batch(fmt):
    B = 65535
    g = gen(66)
    lens = [i % 5 for i in range(B)]
    prefix = prefix_rows(g, 1, 1, 130, [130])
    attn_case(fmt, B, 1, 1, 5, lens, 67, True, seqs=[0, 1, 4, 255, 256, 32767, 32768, 65533, 65534])
    attn_case(fmt, B, 1, 1, 5, lens, 67, True, prefix=prefix, n_prefix=1, max_prefix=130, seqs=[0, 1, 4, 255, 256, 32767, 32768, 65533, 65534])


@pytest.mark.parametrize("view", ["heads first", "tokens last", "every other token", "one token", "one head"])
def test_read_into_views(view):
    B, T, H = (3, 1, 2) if view == "one token" else (3, 10, 1) if view == "one head" else (3, 10, 2)
    st, _ = filled("int8", B, 4, H, 12, [T] * B, 68)
    want = dequantised(st)
    def target():
        if view == "heads first":
            return torch.zeros((B, H, T, 128), dtype=torch.bfloat16, device=DEV).transpose(1, 2)
        if view == "tokens last":
            return torch.zeros((T, H, B, 128), dtype=torch.bfloat16, device=DEV).permute(2, 0, 1, 3)
        if view == "every other token":
            return torch.zeros((B, 2 * T, H, 128), dtype=torch.bfloat16, device=DEV)[:, ::2]
        return torch.zeros((B, T, H, 128), dtype=torch.bfloat16, device=DEV)
    k, v = target(), target()
    st.read(k, v)
    for x, y in zip((k, v), want):
        assert (f64(x) == ref.round_bf16(y[:, :, :T].transpose(0, 2, 1, 3))).all()
    if T > 1:
        one = torch.zeros((B, 1, H, 128), dtype=torch.bfloat16, device=DEV)
        with pytest.raises(gkv.GKVError):
            st.read(one.expand(B, T, H, 128), one.expand(B, T, H, 128))


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("h_q,h_kv,lens", [
    (4, 1, [9999, 0, -1, 5, 20000, 700]), (7, 1, [0, 0, -1, 0, 0, 0]), (4, 2, [1, 9000] + [0] * 18 + [-1, 33, 3000]), (8, 1, [130] * 45 + [8000]),
    (2, 1, [15, 16, 17, 9999]), (1, 1, [9990, 9991]),
])
def test_pieces_go_by_the_lengths(fmt, append, h_q, h_kv, lens):
    """Few units and a long capacity: very uneven lengths, sequences without keys, left out and not fitting."""
    C = 10000
    fits = [min(x, C - 1) for x in lens]
    st, g = filled(fmt, len(lens), h_q, h_kv, C, fits, 71)
    q = randn(g, len(lens), h_q, 128)
    kn, vn = (randn(g, len(lens), h_kv, 128), randn(g, len(lens), h_kv, 128)) if append else (None, None)
    out, lse = torch.full((len(lens), h_q, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((len(lens), h_q), 7.0, device=DEV)
    st.attn(ints(lens), q, out, k_new=kn, v_new=vn, lse=lse)
    skip = [b for b, x in enumerate(lens) if x < 0 or x > C]
    check(st, lens, q, out, lse, append, skip=skip)
    for b in skip:
        assert (out[b] == 7).all() if lens[b] < 0 else torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
    again = torch.empty_like(out)
    if not append:
        st.attn(ints(lens), q, again, max_len=C)
        keep = [b for b in range(len(lens)) if b not in skip]
        assert torch.equal(out[keep], again[keep])


class Some:
    """A few sequences of a store, for the reference."""
    def __init__(self, st, seqs):
        self.fmt, self.h_q, self.h_kv, self.batch = st.fmt, st.h_q, st.h_kv, len(seqs)
        self.k, self.v, self.k_scale, self.v_scale = (None if t is None else t[seqs] for t in (st.k, st.v, st.k_scale, st.v_scale))


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("fmt,B,h_kv,C,long", [
    ("int8", 150, 2, 8300, {3: 8299, 149: 5000}),     # more units than there are places
    ("int4", 330, 1, 8300, {40: 8299, 41: 8000}),     # more sequences than two turns of a warp
    ("e4m3", 40, 2, 17000, {0: 16999, 33: 4001}), ("bf16", 20, 4, 15000, {19: 14999}), ("int4", 37, 3, 16400, {36: 16399}),
])
def test_long_sequences_among_short_ones(fmt, append, B, h_kv, C, long):
    rng = np.random.RandomState(B)
    lens = [int(x) for x in rng.randint(-1, 60, B)]
    for b, n in long.items():
        lens[b] = n
    st, g = filled(fmt, B, 4 * h_kv, h_kv, C, lens, 72)
    q = randn(g, B, 4 * h_kv, 128)
    kn, vn = (randn(g, B, h_kv, 128), randn(g, B, h_kv, 128)) if append else (None, None)
    out, lse = torch.full((B, 4 * h_kv, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((B, 4 * h_kv), 7.0, device=DEV)
    st.attn(ints(lens), q, out, k_new=kn, v_new=vn, lse=lse)
    seqs = sorted(set(long) | set(range(0, B, 9)))
    seqs = [b for b in seqs if lens[b] >= 0]
    check(Some(st, seqs), [lens[b] for b in seqs], q[seqs], out[seqs], lse[seqs], append)
    for b in range(B):
        assert (out[b] == 7).all() if lens[b] < 0 else torch.isfinite(out[b]).all()


def test_a_captured_graph_deals_out_by_the_lengths_it_finds():
    B, C = 12, 12000
    st, g = filled("int8", B, 4, 1, C, [C - 3] * B, 73)
    q, kn, vn = randn(g, B, 4, 128), randn(g, B, 1, 128), randn(g, B, 1, 128)
    out, lse = torch.zeros((B, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((B, 4), device=DEV)
    length = ints([100] * B)
    st.attn(length, q, out, k_new=kn, v_new=vn, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.attn(length, q, out, k_new=kn, v_new=vn, lse=lse)
        length += 1
    for lens in ([100] * B, [11990] + [3] * (B - 1), [-2, 0] + [6000] * (B - 2)):
        out.fill_(7)
        length.copy_(ints(lens))
        graph.replay()
        torch.cuda.synchronize()
        assert length.tolist() == [x + 1 for x in lens]
        check(st, lens, q, out, lse, True, skip=[b for b in range(B) if lens[b] < 0])
        for b in range(B):
            assert (out[b] == 7).all() if lens[b] < 0 else torch.isfinite(out[b]).all()
