"""Key/value stores at the ends of their documented range: tokens and rows at the ends of 32 bits, groups of a 4-bit row that differ by
many powers of two."""
import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
import store_reference as ref
from test_gpu_store import DEV, FORMATS, dequantised, expect_codes, f64, gen, ints, randn, raw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


@pytest.mark.parametrize("fmt", FORMATS)
def test_first_and_count_at_the_ends_of_32_bits(fmt):
    """A count below 0 is none, one above the tokens is all of them, and rows outside the store are left out, however far out; more
    tokens than rows."""
    lo, hi = -2 ** 31, 2 ** 31 - 1
    first = [0, 5, hi, hi - 100, lo, -40, 0, 3]
    count = [lo, -1, hi, 256, hi, 200, hi, lo + 64]
    B, T, H, C = len(first), 256, 2, 96
    x = randn(gen(11), 2, B, T, H, 128)
    st = gkv.KVStore(fmt, batch=B, h_q=4, h_kv=H, capacity=C, device=DEV)
    bufs = [t for t in (st.k, st.v, st.k_scale, st.v_scale) if t is not None]
    for t in bufs:
        t.view(torch.uint8).fill_(0x3A)
    st.write(x[0], x[1], first=ints(first), count=ints(count))
    written = np.zeros((B, C), bool)
    token = np.zeros((B, C), int)
    for b in range(B):
        for t in range(max(0, min(count[b], T))):
            if 0 <= first[b] + t < C:
                written[b, first[b] + t], token[b, first[b] + t] = True, t
    assert written.any(1).tolist() == [False, False, False, False, False, True, True, False]
    for i, (codes, scale) in enumerate(((st.k, st.k_scale), (st.v, st.v_scale))):
        for b in np.flatnonzero(written.any(1)):
            r = np.flatnonzero(written[b])
            want, s = expect_codes(x[i, b, token[b, r]].transpose(0, 1).contiguous(), fmt)
            assert (raw(codes[b])[:, r].reshape(want.shape) == want).all()
            if scale is not None:
                assert (f64(scale[b])[:, r] == s).all()
    for t in bufs:
        assert (raw(t).reshape(B, H, C, -1).transpose(0, 2, 1, 3)[~written] == 0x3A).all()
    out = torch.full((2, B, T, H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    st.read(out[0], out[1], first=ints(first), count=ints(count))
    got = np.zeros((B, T), bool)
    for b in range(B):
        r = np.flatnonzero(written[b])
        got[b, token[b, r]] = True
    assert (f64(out)[:, ~got] == 7.0).all()
    for i in range(2):
        want = f64(x[i])[got]
        if fmt != "bf16":
            want = ref.round_bf16(ref.values(*ref.encode(want, fmt), fmt))
        assert (f64(out[i])[got] == want).all()


# Groups of a 4-bit row differ by powers of two: the rest, one far below it, one far above, and one that differs from key to key.
def rows_of_uneven_groups(g, shape, exponent):
    x = randn(g, *shape)
    x[..., 32:64] *= 2.0 ** -exponent
    x[..., 64:96] *= 2.0 ** (exponent // 3)
    x[..., 96:] *= torch.exp2(torch.randint(-exponent, 1, shape[:-1] + (1,), generator=g, device=DEV).float()).to(torch.bfloat16)
    return x


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("exponent", [12, 30, 48, 96])
@pytest.mark.parametrize("B,H,C,m", [(300, 2, 40, 0), (2, 1, 300, 0), (1, 1, 4000, 0), (3, 2, 9000, 0), (4, 1, 130, 200), (2, 1, 130, 0)],
                         ids=["whole", "cluster", "pieces", "dealt", "prefix", "small"])
def test_groups_of_very_different_size(B, H, C, m, exponent, append):
    """Each group of 32 dimensions is as precise as if it were alone: the tolerance of a group counts that group's values only."""
    g, rng = gen(17 + exponent), np.random.RandomState(exponent)
    Hq = 4 * H
    st = gkv.KVStore("int4", batch=B, h_q=Hq, h_kv=H, capacity=C, device=DEV, n_prefix=1 if m else 0, max_prefix=m)
    lens = rng.randint(0, C, B)
    lens[0], lens[-1] = C - 1, C - 1
    st.write(randn(g, B, C, H, 128), rows_of_uneven_groups(g, (B, C, H, 128), exponent))
    q, out, lse = randn(g, B, Hq, 128), torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=DEV), torch.empty((B, Hq), device=DEV)
    new = dict(k_new=randn(g, B, H, 128), v_new=rows_of_uneven_groups(g, (B, H, 128), exponent)) if append else {}
    kp, vp = randn(g, 1, H, m, 128), rows_of_uneven_groups(g, (1, H, m, 128), exponent)
    st.attn(ints(lens.tolist()), q, out, lse=lse, prefix=gkv.Prefix(kp, vp, [m]) if m else None, **new)
    K, V = dequantised(st)
    lens = lens + append
    out, lse, q, kp, vp = f64(out), f64(lse), f64(q), f64(kp), f64(vp)
    for b in range(B):
        for h in range(H):
            heads, n = slice(4 * h, 4 * h + 4), lens[b]
            for i in range(4):
                d = slice(32 * i, 32 * i + 32)
                pre = (kp[0, h], vp[0, h, :, d]) if m else (None, None)
                if n + m == 0:
                    assert (out[b, heads] == 0).all() and (lse[b, heads] == -np.inf).all()
                    continue
                want, l, tol, ltol = ref.attend(q[b, heads], K[b, h, :n], V[b, h, :n, d], *pre)
                assert (np.abs(out[b, heads, d] - want) <= tol).all(), (b, h, i, np.abs(out[b, heads, d] - want).max() / np.abs(want).max())
                assert (np.abs(lse[b, heads] - l) <= ltol).all()


@pytest.mark.parametrize("rise", [13, 14, 15, 16])           # in units of e: weights of 2^19 to 2^23 relative to the first tiles
@pytest.mark.parametrize("period", [4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 16, 22, 32])
@pytest.mark.parametrize("seqs", [16, 32])
def test_partial_results_of_large_values_add_up(seqs, period, rise):
    """V of 2^96 and logits that are low in the first two of every `period` key tiles and high in the others: where that is how the
    keys are cut into runs, every partial result comes near the end of fp32's range, each of them finite, and so has to be their sum."""
    m, H = 8192, 16
    g = gen(71)
    high = (torch.arange(m // 128, device=DEV) % period >= 2).repeat_interleave(128)
    q = randn(g, 1, 1, 128).expand(seqs, 8 * H, 128).contiguous()
    unit = q[0, 0].float() / q[0, 0].float().square().sum() * 128 ** 0.5
    k = (unit * (high * rise)[:, None]).to(torch.bfloat16).view(1, 1, m, 128).expand(1, H, m, 128).contiguous()
    v = (torch.rand(1, H, m, 128, generator=g, device=DEV) * 2.0 ** 96).to(torch.bfloat16)
    out, lse = torch.empty((seqs, 8 * H, 128), dtype=torch.bfloat16, device=DEV), torch.empty((seqs, 8 * H), device=DEV)
    st = gkv.KVStore("bf16", batch=seqs, h_q=8 * H, h_kv=H, capacity=4, device=DEV, n_prefix=1, max_prefix=m)
    st.attn(ints([0] * seqs), q, out, prefix=gkv.Prefix(k, v, [m]), lse=lse)
    assert torch.isfinite(out).all()
    for h in (0, H - 1):
        hs = slice(8 * h, 8 * h + 8)
        want, l, tol, ltol = ref.attend(f64(q[1, hs]), np.zeros((0, 128)), np.zeros((0, 128)), f64(k[0, h]), f64(v[0, h]), ref.U_BF16)
        assert (np.abs(f64(out[1, hs]) - want) <= tol).all() and (np.abs(f64(lse[1, hs]) - l) <= ltol).all()
