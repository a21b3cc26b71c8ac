"""Caches in pages on the GPU: appending with and without the rotation and reading back (bit-exact against the rotation by itself and the
fp64 reference of the row formats), and decode attention over the pages against the fp64 reference."""
import math

import numpy as np
import pytest
import torch

import pages_reference as pref
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
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def raw(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def plain(rot):
    return [10000.0 ** (-2 * i / rot) for i in range(rot // 2)]


def rotary(kind):
    """None, or (pairs' order, rotated part) of a head of 128."""
    return None if kind is None else gkv.Rotary(plain(kind[1]), interleaved=kind[0] == "neighbours", factor=1.25 if kind[1] == 64 else 1.0, device=DEV)


def deal_pages(seed, lens, page, spare=3, width=None):
    """A table in which every sequence has the pages that it needs, in no order, the other places -1; and the number of pages."""
    need = [max(0, -(-n // page)) for n in lens]
    order = np.random.RandomState(seed).permutation(sum(need) + spare)
    table = np.full((len(lens), width or max(max(need), 1)), -1, np.int64)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def token_first(store, t):
    """[pages][slot][head][...]"""
    return t if store.token_major else t.transpose(1, 2)


def stored(store):
    """The rows' bytes [pages][slot][head][row] and scales (fp64) of K and V."""
    return [(raw(token_first(store, c)).reshape(store.pages, store.page_size, store.h_kv, -1), None if s is None else f64(token_first(store, s)))
            for c, s in ((store.k, store.k_scale), (store.v, store.v_scale))]


def values_of(store):
    """The rows as fp64 [pages][slot][head][128], by the reference's reading of the bytes."""
    got = []
    for codes, scale in ((store.k, store.k_scale), (store.v, store.v_scale)):
        codes = token_first(store, codes)
        if store.fmt == "bf16":
            got.append(f64(codes))
            continue
        s = f64(token_first(store, scale))
        if store.fmt == "int4":
            b = codes.cpu().numpy().astype(np.int64)
            c = np.zeros(b.shape[:-1] + (128,))
            for e in range(128):
                w, i = 4 * (e % 32 // 4) + e // 32, e % 4
                c[..., e] = ((b[..., 2 * w + i // 2] >> (4 * (i % 2))) & 15) - 8
        else:
            c = f64(codes.float())
        got.append(ref.values(c, s, store.fmt))
    return got


def expect_codes(x, fmt):
    """bytes [..., row], scales fp64 [..., groups] of bf16 rows x."""
    if fmt == "bf16":
        return raw(x).reshape(x.shape[:-1] + (256,)), None
    c, s = ref.encode(f64(x), fmt)
    return ref.pack(c, fmt), s


def turned(rot, pos, x):
    """x [batch][tokens][heads][128] as the rotation by itself leaves it."""
    if rot is None:
        return x.contiguous()
    y = torch.empty(x.shape, dtype=x.dtype, device=DEV)
    rot.apply(pos, x, q_out=y)
    return y


# ---------------------------------------------------------------------------------------------- append, read
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,token_major", [(16, False), (16, True), (1, False), (5, True), (24, False), (64, False), (256, True)])
@pytest.mark.parametrize("kind", [None, ("halves", 128), ("halves", 64), ("neighbours", 128), ("neighbours", 44), ("halves", 20), ("halves", 6), ("halves", 96)])
def test_append_and_read(fmt, page, token_major, kind):
    """Ragged counts, runs that begin anywhere, rows outside the table, a strided source: the rows' bytes are those of the rotation by itself and
    the reference's quantisation, all others as they were."""
    B, T, H, Hq, width = 5, 37, 3, 6, -(-64 // page)
    g = gen(3)
    first, count = [0, 27, width * page - 4, 3, -2], [37, 37, 37, 0, 9]       # the last ones reach past both ends
    table, n_pages = deal_pages(1, [width * page] * B, page)
    table[1, width - 1] = -1                                                    # and these have no page
    table[0, 0] = n_pages
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=Hq, h_kv=H, max_batch=B, token_major=token_major, device=DEV)
    for t in (st.k, st.v, st.k_scale, st.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x3A)
    qkv = randn(g, B, T, Hq + 2 * H, 128) * torch.exp2(torch.randint(-20, 20, (B, T, Hq + 2 * H, 1), generator=g, device=DEV).to(torch.bfloat16))
    k, v = qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
    rot = rotary(kind)
    given = kind is not None and kind[1] == 64                                 # positions of their own, or the rows' numbers
    pos = torch.randint(0, 9999, (B, T), generator=g, device=DEV, dtype=torch.int32) if given else ints(first)[:, None] + torch.arange(T, device=DEV, dtype=torch.int32)
    st.append(ints(table), k, v, first=ints(first), count=ints(count), rotary=rot, pos=pos if given else None)
    want = [expect_codes(turned(rot, pos, k), fmt), expect_codes(v.contiguous(), fmt)]
    got = stored(st)
    written = np.zeros((n_pages, page), bool)
    there = np.zeros((B, T), bool)
    for b in range(B):
        for t in range(count[b]):
            r = first[b] + t
            if not 0 <= r < width * page or not 0 <= table[b, r // page] < n_pages:
                continue
            p, s = table[b, r // page], r % page
            written[p, s] = there[b, t] = True
            for (codes, scale), (wc, ws) in zip(got, want):
                assert (codes[p, s] == wc[b, t]).all(), (b, t)
                if scale is not None:
                    assert (scale[p, s] == ws[b, t]).all(), (b, t)
    for t in (st.k, st.v, st.k_scale, st.v_scale):
        if t is not None:
            assert (raw(token_first(st, t)).reshape(n_pages, page, -1)[~written] == 0x3A).all()
    wide = torch.full((2, B, T + 3, H + 1, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    out = wide[:, :, :T, :H]
    st.read(ints(table), out[0], out[1], first=ints(first), count=ints(count))
    vals = values_of(st)
    back = f64(wide)
    for b in range(B):
        for t in range(T):
            for kv in range(2):
                if there[b, t]:
                    r = first[b] + t
                    assert (back[kv, b, t, :H] == ref.round_bf16(vals[kv][table[b, r // page], r % page])).all()
                else:
                    assert (back[kv, b, t, :H] == 7).all()
    assert (back[:, :, T:] == 7).all() and (back[:, :, :, H:] == 7).all()


@pytest.mark.parametrize("h_kv", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17])
@pytest.mark.parametrize("kind", [("halves", 128), ("neighbours", 128)])
def test_append_with_any_number_of_heads(h_kv, kind):
    """A CTA's items touch different numbers of runs; the fused append leaves what rotating and then storing does."""
    B, T = 2, 83
    g = gen(h_kv)
    k, v = randn(g, B, T, h_kv, 128), randn(g, B, T, h_kv, 128)
    rot = rotary(kind)
    table, n_pages = deal_pages(2, [T] * B, 16)
    st = gkv.PagedStore("e4m3", pages=n_pages, page_size=16, h_q=h_kv, h_kv=h_kv, max_batch=B, device=DEV)
    st.append(ints(table), k, v, rotary=rot)
    flat = gkv.KVStore("e4m3", batch=B, h_q=h_kv, h_kv=h_kv, capacity=T, device=DEV)
    flat.write(turned(rot, torch.arange(T, device=DEV, dtype=torch.int32).expand(B, T), k), v)
    for a, b in ((st.k, flat.k), (st.v, flat.v), (st.k_scale, flat.k_scale), (st.v_scale, flat.v_scale)):
        rows = a.view(torch.uint8)[ints(table).long()].transpose(1, 2).flatten(2, 3)[:, :, :T]
        assert torch.equal(rows, b.view(torch.uint8))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("h_kv", [3, 4, 8, 12])
@pytest.mark.parametrize("kind", [None, ("halves", 128), ("halves", 64), ("halves", 16), ("halves", 20), ("neighbours", 128), ("neighbours", 64), ("neighbours", 24), ("neighbours", 44)])
def test_append_of_many_rows(fmt, h_kv, kind):
    """As many as take the wider runs, every way of turning them: the bytes that rotating and then storing leaves, and all others as they were."""
    B, T, cap = 3, 307, 320
    g = gen(7)
    first, count = [0, 13, 5], [307, 290, 1]
    kv = randn(g, B, T, 2 * h_kv, 128) * torch.exp2(torch.randint(-20, 20, (B, T, 2 * h_kv, 1), generator=g, device=DEV).to(torch.bfloat16))
    kv[0, 40, 0, 5], kv[0, 41, h_kv, 77], kv[1, 2, 1, 100] = float("nan"), float("inf"), float("-inf")      # their rows are not finite
    k, v = kv[:, :, :h_kv], kv[:, :, h_kv:]
    rot = rotary(kind)
    table, n_pages = deal_pages(3, [cap] * B, 16)
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=16, h_q=h_kv, h_kv=h_kv, max_batch=B, device=DEV)
    flat = gkv.KVStore(fmt, batch=B, h_q=h_kv, h_kv=h_kv, capacity=cap, device=DEV)
    for t in (st.k, st.v, st.k_scale, st.v_scale, flat.k, flat.v, flat.k_scale, flat.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x3A)
    st.append(ints(table), k, v, first=ints(first), count=ints(count), rotary=rot)
    pos = ints(first)[:, None] + torch.arange(T, device=DEV, dtype=torch.int32)
    flat.write(turned(rot, pos, k), v.contiguous(), first=ints(first), count=ints(count))
    for a, b in ((st.k, flat.k), (st.v, flat.v), (st.k_scale, flat.k_scale), (st.v_scale, flat.v_scale)):
        if a is not None:
            rows = a.view(torch.uint8)[ints(table).long()].transpose(1, 2).flatten(2, 3)[:, :, :cap]
            assert torch.equal(rows, b.view(torch.uint8))


def test_no_tokens_do_nothing():
    st = gkv.PagedStore("int8", pages=2, page_size=16, h_q=4, h_kv=2, max_batch=1, device=DEV)
    x = torch.zeros(1, 0, 2, 128, dtype=torch.bfloat16, device=DEV)
    st.append(ints([[0]]), x, x.clone())
    st.read(ints([[0]]), x, x.clone())


# ---------------------------------------------------------------------------------------------- attention
def filled(fmt, seed, lens, page, h_q, h_kv, token_major=False, width=None, spare=3, scale=1.0):
    """A store whose sequences have their rows, every other row NaN (in its data or its scales), its table, and room for one row more."""
    g = gen(seed)
    table, n_pages = deal_pages(seed, [max(n, 0) + 1 for n in lens], page, spare, width)
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=len(lens), token_major=token_major, device=DEV)
    for t in (st.k, st.v) if fmt == "bf16" else (st.k_scale, st.v_scale):
        t.fill_(math.nan)
    if fmt != "bf16":
        st.k.view(torch.uint8).fill_(0x7F), st.v.view(torch.uint8).fill_(0x7F)
    T = max(max(lens), 1)
    k, v = randn(g, len(lens), T, h_kv, 128) * scale, randn(g, len(lens), T, h_kv, 128)
    st.append(ints(table), k.to(torch.bfloat16), v, count=ints(lens))
    return st, table, g


def expect(st, table, length, q, rows, positions=None):
    """Outputs, lse and tolerances of sequences that attend to their first rows[i] rows as they stand in the store; q as it attends."""
    K, V = values_of(st)
    B, h_q = q.shape[:2]
    g = h_q // st.h_kv
    out, lse, to, tl = np.zeros((B, h_q, 128)), np.zeros((B, h_q)), np.zeros((B, h_q, 128)), np.zeros((B, h_q))
    for b in range(B):
        p, s = pref.pool_rows(table[b], st.page_size, np.arange(max(rows[b], 0)))
        for h in range(st.h_kv):
            sl = slice(h * g, (h + 1) * g)
            out[b, sl], lse[b, sl], to[b, sl], tl[b, sl] = ref.attend(f64(q[b, sl]), K[p, s, h], V[p, s, h],
                                                                      weight_unit=ref.U_BF16 if st.fmt == "bf16" else ref.U_F16)
    return out, lse, to, tl


def close(got, want, tol):
    """NaN and infinities in the same places, the rest within the tolerance."""
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    assert ok.all(), (np.abs(got - want)[~ok].max(), np.argwhere(~ok)[:3])


def run(st, table, lens, q, k_new=None, v_new=None, rot=None, pos=None, max_len=0):
    out = torch.full((len(lens), st.h_q, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((len(lens), st.h_q), 9.0, dtype=torch.float32, device=DEV)
    st.attn(ints(table), ints(lens), q, out, k_new=k_new, v_new=v_new, rotary=rot, pos=pos, lse=lse, max_len=max_len)
    return out, lse


LENS = [0, 1, 15, 16, 17, 31, 32, 63, 64, 65, 127, 200, 333, -1, 5]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,token_major,h_q,h_kv", [(16, False, 8, 1), (16, True, 6, 2), (1, False, 7, 1), (5, False, 4, 4), (24, True, 28, 4), (64, False, 16, 2), (256, False, 3, 1)])
@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("kind", [None, ("halves", 128), ("neighbours", 64)])
def test_attention(fmt, page, token_major, h_q, h_kv, append, kind):
    st, table, g = filled(fmt, 20, LENS, page, h_q, h_kv, token_major)
    B = len(LENS)
    qkv = randn(g, B, h_q + 2 * h_kv, 128)                        # slices of one projection's output
    q, k_new, v_new = qkv[:, :h_q], qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:]
    rot = rotary(kind)
    pos = ints(np.arange(B) * 1000 + 7) if kind is not None and kind[1] == 64 else None
    before = stored(st)
    out, lse = run(st, table, LENS, q, k_new if append else None, v_new if append else None, rot, pos)
    at = (pos if pos is not None else ints([n if append else n - 1 for n in LENS]))[:, None]
    written = np.zeros((st.pages, page), bool)
    after = stored(st)
    if append:                                                     # the new rows' bits, and nothing else
        want = [expect_codes(turned(rot, at, k_new[:, None])[:, 0], fmt), expect_codes(v_new.contiguous(), fmt)]
        for b, n in enumerate(LENS):
            if n >= 0:
                p, s = table[b, n // page], n % page
                written[p, s] = True
                for (codes, scale), (wc, ws) in zip(after, want):
                    assert (codes[p, s] == wc[b]).all(), b
                    assert scale is None or (scale[p, s] == ws[b]).all(), b
    for (c0, s0), (c1, s1) in zip(before, after):
        assert (c0[~written] == c1[~written]).all() and (s0 is None or np.array_equal(s0[~written], s1[~written], equal_nan=True))
    rows = [n + 1 if append and n >= 0 else n for n in LENS]
    eo, el, to, tl = expect(st, table, LENS, turned(rot, at, q[:, None])[:, 0], rows)
    for b, n in enumerate(LENS):
        if n < 0:
            assert (out[b] == 9).all() and (lse[b] == 9).all()      # left out
        else:
            close(f64(out[b]), eo[b], to[b])
            close(f64(lse[b]), el[b], tl[b])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens,h_q,h_kv", [([2000], 8, 1), ([700], 28, 4), ([9000], 7, 1), ([40000], 8, 2), ([5000, 3], 8, 2), ([12000, 0, 100, 1], 4, 1),
                                           ([4100] * 6, 4, 1), ([300] * 40, 28, 4), ([70] * 400, 8, 2)])
def test_work_spread_over_the_length(fmt, lens, h_q, h_kv):
    """Clusters, pieces that meet in the workspace, whole units; lengths far apart; the longest length given or not."""
    st, table, g = filled(fmt, 21, lens, 16, h_q, h_kv)
    B = len(lens)
    q, k_new, v_new = randn(g, B, h_q, 128), randn(g, B, h_kv, 128), randn(g, B, h_kv, 128)
    results = []
    for max_len in (max(lens), 0):
        out, lse = run(st, table, lens, q, k_new, v_new, max_len=max_len)
        again = run(st, table, lens, q, k_new, v_new, max_len=max_len)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
        results.append((f64(out), f64(lse)))
    picked = sorted({0, B // 2, B - 1})
    eo, el, to, tl = expect(st, table[picked], None, q[picked], [lens[b] + 1 for b in picked])
    for out, lse in results:
        close(out[picked], eo, to)
        close(lse[picked], el, tl)
    # the two plans are both within the tolerance of the same number
    close(results[0][0], results[1][0], 2 * to.max() + 2.0 ** -7 * np.abs(results[1][0]))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", [("halves", 20), ("halves", 6), ("halves", 96), ("neighbours", 44), ("neighbours", 2), ("halves", 126)])
@pytest.mark.parametrize("lens", [[70, 0, 33], [6000, 17, 2100]])
def test_parts_of_a_head(fmt, kind, lens):
    """Every way in which words and single elements are turned, in the short form and the one of equal shares; at the rows' numbers."""
    st, table, g = filled(fmt, 40, lens, 16, 7, 1)
    q, k_new, v_new = randn(g, 3, 7, 128), randn(g, 3, 1, 128), randn(g, 3, 1, 128)
    rot = rotary(kind)
    out, lse = run(st, table, lens, q, k_new, v_new, rot)
    at = ints(lens)[:, None]
    for (codes, scale), (wc, ws) in zip(stored(st), [expect_codes(turned(rot, at, k_new[:, None])[:, 0], fmt), expect_codes(v_new, fmt)]):
        for b, n in enumerate(lens):
            p, s = table[b, n // 16], n % 16
            assert (codes[p, s] == wc[b]).all() and (scale is None or (scale[p, s] == ws[b]).all())
    eo, el, to, tl = expect(st, table, lens, turned(rot, at, q[:, None])[:, 0], [n + 1 for n in lens])
    close(f64(out), eo, to)
    close(f64(lse), el, tl)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page,token_major,h_kv", [(16, False, 2), (32, False, 1), (48, False, 2), (64, True, 2), (1, False, 1), (7, True, 2)])
@pytest.mark.parametrize("append", [False, True])
def test_equal_shares(fmt, page, token_major, h_kv, append):
    """Long calls: units that several warps share, that one has to itself and that have no rows; ends of a page, a tile, a step and a share; left out,
    empty and unfitting sequences among them; everything behind the ends NaN."""
    lens = [4095, -1, 0, 1, 31, 32, 33, 2047, 2 ** 31 - 1, 900, 16, 4096, 15, 5000]
    have = [n if n < 10000 else 0 for n in lens]
    st, table, g = filled(fmt, 41, have, page, 4 * h_kv, h_kv, token_major)
    B = len(lens)
    qkv = randn(g, B, 6 * h_kv, 128)
    q, k_new, v_new = qkv[:, :4 * h_kv], qkv[:, 4 * h_kv:5 * h_kv], qkv[:, 5 * h_kv:]
    before = stored(st)
    out, lse = run(st, table, lens, q, k_new if append else None, v_new if append else None)
    written = np.zeros((st.pages, page), bool)
    want = [expect_codes(x.contiguous(), fmt) for x in (k_new, v_new)]
    after = stored(st)
    for b, n in enumerate(lens):
        if append and 0 <= n < 10000:
            p, s = table[b, n // page], n % page
            written[p, s] = True
            for (codes, scale), (wc, ws) in zip(after, want):
                assert (codes[p, s] == wc[b]).all() and (scale is None or (scale[p, s] == ws[b]).all())
    for (c0, s0), (c1, s1) in zip(before, after):
        assert (c0[~written] == c1[~written]).all() and (s0 is None or np.array_equal(s0[~written], s1[~written], equal_nan=True))
    eo, el, to, tl = expect(st, table, lens, q, [n + append if 0 <= n < 10000 else 0 for n in lens])
    for b, n in enumerate(lens):
        if n < 0:
            assert (out[b] == 9).all() and (lse[b] == 9).all()
        elif n > 10000:
            assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
        else:
            close(f64(out[b]), eo[b], to[b])
            close(f64(lse[b]), el[b], tl[b])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("batch,h_kv,longest", [(200, 8, 200), (1100, 1, 130), (2049, 1, 300), (40, 4, 1500), (300, 8, 500)])
def test_many_sequences(fmt, batch, h_kv, longest):
    """More sequences than a warp keeps lengths of, than the merge is made for, and units far more than warps; the results of a few."""
    rng = np.random.RandomState(batch)
    lens = rng.randint(0, longest + 1, batch)
    lens[rng.randint(batch)] = longest
    st, table, g = filled(fmt, 42, lens.tolist(), 16, 2 * h_kv, h_kv)
    q, k_new, v_new = randn(g, batch, 2 * h_kv, 128), randn(g, batch, h_kv, 128), randn(g, batch, h_kv, 128)
    out, lse = run(st, table, lens, q, k_new, v_new, max_len=longest)
    picked = sorted({0, 31, 32, 127, 128, batch // 2, batch - 1} & set(range(batch)))
    eo, el, to, tl = expect(st, table[picked], None, q[picked], [lens[b] + 1 for b in picked])
    close(f64(out[picked]), eo, to)
    close(f64(lse[picked]), el, tl)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_table_far_wider_than_the_lengths(fmt):
    """As in a captured step that leaves max_len to the table: most CTAs have nothing to do."""
    lens = [40, 0, 1000]
    st, table, g = filled(fmt, 22, lens, 16, 8, 2, width=4096)
    q = randn(g, 3, 8, 128)
    out, lse = run(st, table, lens, q)
    eo, el, to, tl = expect(st, table, lens, q, lens)
    close(f64(out), eo, to)
    close(f64(lse), el, tl)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("append", [False, True])
def test_lengths_that_do_not_fit(fmt, append):
    lens = [48, 49, 47, 2 ** 31 - 1]
    st, table, g = filled(fmt, 23, [47] * 4, 16, 4, 2)
    q, k_new, v_new = randn(g, 4, 4, 128), randn(g, 4, 2, 128), randn(g, 4, 2, 128)
    assert table.shape[1] == 3
    st.append(ints(table), k_new[:, None], v_new[:, None], first=ints([47] * 4))
    before = stored(st)
    out, lse = run(st, table, lens, q, k_new if append else None, v_new if append else None)
    fits = [not append, False, True, False]
    after = stored(st)
    p = table[2, 2]
    for (c0, s0), (c1, s1) in zip(before, after):
        same = (c0 == c1).all((-1, -2))
        same[p, 15] = True
        assert same.all()
    eo, el, to, tl = expect(st, table, lens, q, [48, 0, 48 if append else 47, 0])
    for b in range(4):
        if fits[b]:
            close(f64(out[b]), eo[b], to[b])
            close(f64(lse[b]), el[b], tl[b])
        else:
            assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [16, 5, 64])
@pytest.mark.parametrize("bad", [-1, "pages", 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("long", [False, True])
def test_places_without_a_page(fmt, page, bad, long):
    """They make their own sequence NaN and touch nothing; the new row of one is not written."""
    lens = [9000, 130, 5000, 77] if long else [100, 130, 64, 77]
    st, table, g = filled(fmt, 24, lens, page, 8, 2)
    bad = st.pages if bad == "pages" else bad
    table[0, lens[0] // 2 // page] = bad           # in the middle
    table[2, lens[2] // page] = bad                # the new row's
    q, k_new, v_new = randn(g, 4, 8, 128), randn(g, 4, 2, 128), randn(g, 4, 2, 128)
    before = stored(st)
    out, lse = run(st, table, lens, q, k_new, v_new)
    written = np.zeros((st.pages, page), bool)
    for b in (0, 1, 3):
        written[table[b, lens[b] // page], lens[b] % page] = True
    for (c0, s0), (c1, s1) in zip(before, stored(st)):
        assert (c0[~written] == c1[~written]).all() and (s0 is None or np.array_equal(s0[~written], s1[~written], equal_nan=True))
    for b in (0, 2):
        assert torch.isnan(out[b]).all() and torch.isnan(lse[b]).all()
    eo, el, to, tl = expect(st, table[[1, 3]], None, q[[1, 3]], [lens[1] + 1, lens[3] + 1])
    close(f64(out[[1, 3]]), eo, to)
    close(f64(lse[[1, 3]]), el, tl)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_shared_by_sequences(fmt):
    """Several sequences begin with the same pages and go on with their own."""
    lens = [64 + n for n in (0, 5, 16, 40)]
    st, table, g = filled(fmt, 25, lens, 16, 8, 2)
    table[1:, :4] = table[0, :4]
    q, k_new, v_new = randn(g, 4, 8, 128), randn(g, 4, 2, 128), randn(g, 4, 2, 128)
    out, lse = run(st, table, lens, q, k_new, v_new)
    eo, el, to, tl = expect(st, table, lens, q, [n + 1 for n in lens])
    close(f64(out), eo, to)
    close(f64(lse), el, tl)


def test_large_logits_and_keys_that_count_for_nothing():
    """Maxima that rise along the row, logits of -infinity at its start, and everywhere."""
    lens = [300, 300, 40]
    st, table, g = filled("bf16", 26, lens, 16, 8, 2)
    q = randn(g, 3, 8, 128).abs() + 0.5
    K = token_first(st, st.k)
    for r in range(300):
        p, s = table[0, r // 16], r % 16
        K[p, s] = K[p, s] * 0.01 * r
        if r < 100:
            K[table[1, r // 16], s, :, 5] = -math.inf
    for r in range(40):
        K[table[2, r // 16], r % 16, :, 9] = -math.inf
    out, lse = run(st, table, lens, q)
    eo, el, to, tl = expect(st, table[:1], None, q[:1], [300])
    close(f64(out[:1]), eo, to)
    close(f64(lse[:1]), el, tl)
    Kv, V = values_of(st)
    p, s = pref.pool_rows(table[1], 16, np.arange(100, 300))
    for h in range(2):
        eo, el, to, tl = ref.attend(f64(q[1, 4 * h:4 * h + 4]), Kv[p, s, h], V[p, s, h], weight_unit=ref.U_BF16)
        close(f64(out[1, 4 * h:4 * h + 4]), eo, to)
        close(f64(lse[1, 4 * h:4 * h + 4]), el, tl)
    assert (out[2] == 0).all() and (lse[2] == -math.inf).all()


def test_nan_and_infinity_in_a_new_row_and_in_v():
    lens = [50, 50, 50]
    st, table, g = filled("e4m3", 27, lens, 16, 8, 2)
    q, k_new, v_new = randn(g, 3, 8, 128), randn(g, 3, 2, 128), randn(g, 3, 2, 128)
    k_new[0, 0, 3] = math.inf                      # the group's scale becomes NaN
    v_new[1, 1, 7] = math.nan
    out, lse = run(st, table, lens, q, k_new, v_new)
    assert torch.isnan(out[0, :4]).all() and torch.isnan(lse[0, :4]).all() and torch.isfinite(out[0, 4:]).all()
    assert torch.isfinite(out[1, :4]).all() and torch.isnan(out[1, 4:]).all() and torch.isfinite(out[2]).all()


@pytest.mark.parametrize("fmt,rows", [("bf16", 18_000_000), ("int4", 70_000_000)])
def test_rows_far_into_a_large_pool(fmt, rows):
    """Rows behind 4 GB of codes (and, with 4 bits, behind 2^26 rows): written, read back and attended to at the pool's end."""
    page, n_pages = 64, rows // 64
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=4, h_kv=1, max_batch=2, device=DEV)
    assert st.k.numel() * st.k.element_size() > 2 ** 32
    g = gen(28)
    lens = [200, 130]
    table = np.array([[n_pages - 1, 0, n_pages - 2, n_pages // 2], [n_pages - 3, n_pages - 4, 1, -1]])
    k, v = randn(g, 2, 200, 1, 128), randn(g, 2, 200, 1, 128)
    st.append(ints(table), k, v, count=ints(lens), rotary=(rot := gkv.Rotary(plain(128), device=DEV)))
    back = torch.zeros(2, 2, 200, 1, 128, dtype=torch.bfloat16, device=DEV)
    st.read(ints(table), back[0], back[1], count=ints(lens))
    kr = turned(rot, torch.arange(200, device=DEV, dtype=torch.int32).expand(2, 200), k)
    q = randn(g, 2, 4, 128)
    out, lse = run(st, table, lens, q)
    for b, n in enumerate(lens):
        rows = []
        for x, y in ((kr[b, :n, 0], back[0, b, :n, 0]), (v[b, :n, 0], back[1, b, :n, 0])):
            vals = f64(x) if fmt == "bf16" else ref.values(*ref.encode(f64(x), fmt), fmt)
            assert (f64(y) == ref.round_bf16(vals)).all()
            rows.append(vals)
        eo, el, to, tl = ref.attend(f64(q[b]), *rows, weight_unit=ref.U_BF16 if fmt == "bf16" else ref.U_F16)
        close(f64(out[b]), eo, to)
        close(f64(lse[b]), el, tl)


# ---------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", [("halves", 128), ("neighbours", 32)])
def test_prompts_and_decode_steps(fmt, kind):
    """Prompts appended, then decode steps that append and attend in one call, against the rotation, the store's write and its attention one
    by one: the cache has the same bits, outputs agree within the tolerance of the same number."""
    B, h_q, h_kv, prompt, steps, page = 3, 8, 2, [50, 1, 17], 20, 16
    g = gen(30)
    rot = rotary(kind)
    table, n_pages = deal_pages(5, [n + steps for n in prompt], page)
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=B, device=DEV)
    flat = gkv.KVStore(fmt, batch=B, h_q=h_q, h_kv=h_kv, capacity=80, device=DEV)
    k, v = randn(g, B, 50, h_kv, 128), randn(g, B, 50, h_kv, 128)
    pos = torch.arange(50, device=DEV, dtype=torch.int32).expand(B, 50)
    st.append(ints(table), k, v, count=ints(prompt), rotary=rot)
    flat.write(turned(rot, pos, k), v, count=ints(prompt))
    length = ints(prompt)
    tab = ints(table)
    for step in range(steps):
        q, k1, v1 = randn(g, B, h_q, 128), randn(g, B, h_kv, 128), randn(g, B, h_kv, 128)
        out, out2 = torch.empty_like(q), torch.empty_like(q)
        lse, lse2 = torch.empty(2, B, h_q, device=DEV)
        st.attn(tab, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
        qr, kr = turned(rot, length[:, None], q[:, None])[:, 0], turned(rot, length[:, None], k1[:, None])[:, 0]
        flat.attn(length, qr, out2, k_new=kr, v_new=v1, lse=lse2)
        length += 1
        eo, el, to, tl = expect(st, table, None, qr, [n + step + 1 for n in prompt])
        close(f64(out), eo, to)
        close(f64(out2), eo, to)
        close(f64(lse), el, tl)
    for a, b in ((st.k, flat.k), (st.v, flat.v), (st.k_scale, flat.k_scale), (st.v_scale, flat.v_scale)):
        if a is not None:
            rows = a.view(torch.uint8)[tab.long().clamp(min=0)].transpose(1, 2).flatten(2, 3)
            for i, n in enumerate(prompt):
                assert torch.equal(rows[i, :, :n + steps], b.view(torch.uint8)[i, :, :n + steps])


def test_a_captured_step_replayed_while_lengths_and_tables_grow():
    B, h_q, h_kv, page = 3, 8, 2, 16
    g = gen(31)
    rot = rotary(("halves", 128))
    st = gkv.PagedStore("int8", pages=40, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=B, device=DEV)
    two = gkv.PagedStore("int8", pages=40, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=B, device=DEV)
    order = np.random.RandomState(3).permutation(40)
    table = torch.full((B, 12), -1, dtype=torch.int32, device=DEV)
    length = ints([0, 14, 31])
    used = 0

    def grow():
        nonlocal used
        for b, n in enumerate(length.tolist()):
            for p in range(n // page + 1):
                if table[b, p] < 0:
                    table[b, p] = int(order[used])
                    used += 1

    grow()
    q, k1, v1 = randn(g, B, h_q, 128), randn(g, B, h_kv, 128), randn(g, B, h_kv, 128)
    first = randn(g, 2, B, 31, h_kv, 128)
    for s in (st, two):
        s.append(table, first[0], first[1], count=length, rotary=rot)
    out, lse = torch.zeros_like(q), torch.zeros(B, h_q, device=DEV)
    st.attn(table, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)          # not captured: modules are loaded
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.attn(table, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
    for _ in range(40):
        q.copy_(randn(g, B, h_q, 128)), k1.copy_(randn(g, B, h_kv, 128)), v1.copy_(randn(g, B, h_kv, 128))
        graph.replay()
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        two.attn(table, length, q, o2, k_new=k1, v_new=v1, rotary=rot, lse=l2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        length += 1
        grow()
    assert torch.equal(st.k.view(torch.uint8)[table[table >= 0].long()][:, :, 0], two.k.view(torch.uint8)[table[table >= 0].long()][:, :, 0])


@pytest.mark.parametrize("fmt", ["bf16", "int4"])
def test_long_captured_steps_that_share_a_workspace(fmt):
    """Two stores, each with a captured long step, in one workspace: replayed in turn while their lengths change, from a few rows to many."""
    B, h_q, h_kv = 2, 8, 2
    rot = rotary(("halves", 128))
    g = gen(50)
    stores, graphs, calls = [], [], []
    for i in range(2):
        st, table, _ = filled(fmt, 51 + i, [5000, 5000], 16, h_q, h_kv)
        if i:
            st = gkv.PagedStore(fmt, pages=st.pages, page_size=16, h_q=h_q, h_kv=h_kv, max_batch=B, buffers=[t for t in (st.k, st.v, st.k_scale, st.v_scale) if t is not None],
                                workspace=stores[0].workspace)
            assert st.workspace is stores[0].workspace
        stores.append(st)
        q, k1, v1, length = randn(g, B, h_q, 128), randn(g, B, h_kv, 128), randn(g, B, h_kv, 128), ints([5000, 4000])
        out, lse, tab = torch.zeros_like(q), torch.zeros(B, h_q, device=DEV), ints(table)
        st.attn(tab, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            st.attn(tab, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
        graphs.append(graph)
        calls.append((tab, length, q, out, k1, v1, lse, table))
    for lens in ([4999, 20], [0, 0], [1, 4096], [-1, 3000], [300, 4000]):
        for st, graph, (tab, length, q, out, k1, v1, lse, table) in zip(stores, graphs, calls):
            length.copy_(ints(lens))
            q.copy_(randn(g, B, h_q, 128))
            graph.replay()
            at = length[:, None]
            eo, el, to, tl = expect(st, table, lens, turned(rot, at, q[:, None])[:, 0], [n + 1 for n in lens])
            for b, n in enumerate(lens):
                if n >= 0:
                    close(f64(out[b]), eo[b], to[b])
                    close(f64(lse[b]), el[b], tl[b])


def test_two_stores_on_two_streams():
    g = gen(32)
    made = [filled("bf16", 33 + i, [3000, 20, 700], 16, 8, 2) for i in range(2)]
    qs = [randn(g, 3, 8, 128) for _ in range(2)]
    want = [run(st, table, [3000, 20, 700], q) for (st, table, _), q in zip(made, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = []
        for s, (st, table, _), q in zip(streams, made, qs):
            with torch.cuda.stream(s):
                got.append(run(st, table, [3000, 20, 700], q))
        torch.cuda.synchronize()
        for (o, l), (o2, l2) in zip(got, want):
            assert torch.equal(o, o2) and torch.equal(l, l2)


def test_tensors_that_are_refused():
    st = gkv.PagedStore("bf16", pages=4, page_size=16, h_q=4, h_kv=2, max_batch=2, device=DEV)
    tab, n = torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    k, q, k1 = (torch.zeros(*s, dtype=torch.bfloat16, device=DEV) for s in ((2, 3, 2, 128), (2, 4, 128), (2, 2, 128)))
    small = gkv.Rotary(plain(32), head_dim=64, device=DEV)
    for args, kw in (((tab.long(), k, k.clone()), {}), ((tab[0], k, k.clone()), {}), ((tab.cpu(), k, k.clone()), {}), ((tab[:1], k, k.clone()), {}), ((tab.t(), k, k.clone()), {}),
                     ((tab, k.float(), k.clone()), {}), ((tab, k, k[:, :2]), {}), ((tab, k, k.transpose(1, 2)), {}), ((tab, k, k.clone()), dict(first=n.long())),
                     ((tab, k, k.clone()), dict(count=n[:1])), ((tab, k, k.clone()), dict(rotary=small)), ((tab, k, k.clone()), dict(pos=n)),
                     ((tab, k, k.clone()), dict(pos=tab)), ((None, k, k.clone()), {})):
        with pytest.raises(ValueError):
            st.append(*args, **kw)
    out = torch.zeros_like(q)
    for args, kw in (((tab.long(), n, q, out), {}), ((tab, n.long(), q, out), {}), ((tab, n[:1], q, out), {}), ((tab, n, q.float(), out), {}), ((tab, n, q[:, :2], out), {}),
                     ((tab, n, q, out.float()), {}), ((tab, n, q, torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV)[:, ::2]), {}), ((tab, n, q, out), dict(lse=n)),
                     ((tab, n, torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV)[:, ::2], out), {}), ((tab, n, q, out), dict(k_new=k1[:1], v_new=k1)),
                     ((tab, n, q, out), dict(k_new=k1, v_new=torch.zeros(2, 3, 128, dtype=torch.bfloat16, device=DEV)[:, :2])), ((tab, n, q, out), dict(rotary=small)),
                     ((tab, n, q, out), dict(pos=n.long())), ((torch.zeros(3, 2, dtype=torch.int32, device=DEV), ints([0, 0, 0]), torch.zeros(3, 4, 128, dtype=torch.bfloat16, device=DEV),
                                                               torch.zeros(3, 4, 128, dtype=torch.bfloat16, device=DEV)), {})):
        with pytest.raises(ValueError):
            st.attn(*args, **kw)
    for ws in (torch.zeros(100, dtype=torch.uint8, device=DEV), st.workspace[::2], st.workspace.cpu(), st.workspace.to(torch.int8)):
        with pytest.raises(ValueError):
            gkv.PagedStore("bf16", pages=4, page_size=16, h_q=4, h_kv=2, max_batch=2, buffers=(st.k, st.v), workspace=ws)
    for args, kw in (((tab, n, q, out), dict(k_new=k1)), ((tab, n, q, out), dict(v_new=k1)), ((tab, n, q, out), dict(max_len=33)), ((tab, n, q, out), dict(max_len=-1)),
                     ((tab[:, :0], n, q, out), {})):
        with pytest.raises(gkv.GKVError):
            st.attn(*args, **kw)
    assert not out.any()
