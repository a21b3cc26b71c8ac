"""Rotations and caches in pages on the GPU at the ends of what their description allows."""
import numpy as np
import pytest
import torch

import pages_reference as pref
import paper_2512_00504_b200 as gkv
from test_gpu_pages import deal_pages, randn as rows
from test_gpu_rotary import DEV, check, gen, ints, plain, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


# ---------------------------------------------------------------------------------------------- rotation
@pytest.mark.parametrize("batch,tokens,heads", [(3, 33, 2), (3000, 3, 1)])       # a token a block; several
def test_counts_at_the_lower_end_of_their_range(batch, tokens, heads):
    """A count below 0 leaves the whole sequence as it was, however far below: every block of it, the first and the others."""
    g = gen(60)
    q = randn(g, "bf16", batch, tokens, heads, 128)
    pos = torch.arange(tokens, device=DEV, dtype=torch.int32).expand(batch, tokens)
    count = np.array([-2 ** 31, -2 ** 31 + 1, -1, 0, 1, tokens, 2 ** 31 - 1])[np.arange(batch) % 7]
    count[-1] = -2 ** 31
    rot = gkv.Rotary(plain(128), device=DEV)
    wide = torch.full((batch + 1, tokens, heads, 128), 2.5, device=DEV, dtype=torch.bfloat16)      # and the sequence behind the last
    rot.apply(pos, q, q_out=wide[:batch], count=ints(count))
    turned = torch.from_numpy(np.arange(tokens)[None, :] < count[:, None]).to(DEV)
    assert (wide[:batch][~turned] == 2.5).all() and (wide[batch] == 2.5).all()
    y = wide[:batch].clone()
    y[~turned] = 0
    q[~turned] = 0
    check(rot, "bf16", pos, q, y)


# ---------------------------------------------------------------------------------------------- attention
def cache(fmt, seed, lens, page, h_q, h_kv, token_major=False):
    """Pages full of rows, some of them of sequences of these lengths (and one row more), and their table."""
    table, n_pages = deal_pages(seed, [max(n, 0) + 1 for n in lens], page)
    st = gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=len(lens), token_major=token_major, device=DEV)
    g = gen(seed)
    every = torch.arange(n_pages, dtype=torch.int32, device=DEV)[:, None]
    st.append(every, rows(g, n_pages, page, h_kv, 128), rows(g, n_pages, page, h_kv, 128))
    return st, table, g


@pytest.mark.parametrize("fmt,page,token_major", [("bf16", 16, False), ("bf16", 5, False), ("e4m3", 64, False), ("e4m3", 16, True), ("int8", 16, False),
                                                  ("int4", 32, False), ("int4", 48, False), ("int4", 7, False)])
def test_waits_that_are_taken_for_expired(fmt, page, token_major):
    """Every warp gives up at its first, second .. step: no number comes out where one is missing, new rows are appended as ever, and the call
    after that is right. (Here a warp has four steps, so that none is left to a step of five.)"""
    lens, h_q, h_kv = [5000, 3001], 8, 2
    st, table, g = cache(fmt, 61, lens, page, h_q, h_kv, token_major)
    tab, n = ints(table), ints(lens)
    q, k1, v1 = rows(g, 2, h_q, 128), rows(g, 2, h_kv, 128), rows(g, 2, h_kv, 128)
    buffers = [t for t in (st.k, st.v, st.k_scale, st.v_scale) if t is not None]
    before = [t.view(torch.uint8).clone() for t in buffers]
    out, lse = torch.zeros_like(q), torch.zeros(2, h_q, device=DEV)
    st.attn(tab, n, q, out, k_new=k1, v_new=v1, lse=lse)
    after = [t.view(torch.uint8).clone() for t in buffers]
    assert torch.isfinite(out).all()
    for step in (0, 1, 2, 3, 4, 3, 0):
        for t, b in zip(buffers, before):
            t.view(torch.uint8).copy_(b)
        o, l = torch.zeros_like(out), torch.zeros_like(lse)
        gkv.gkv_selftest_pages_wait(st, step, tab, n, q, o, k_new=k1, v_new=v1, lse=l)
        if step < 4:
            assert torch.isnan(o).all() and torch.isnan(l).all()
        else:
            assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(t.view(torch.uint8), a) for t, a in zip(buffers, after))
        o, l = torch.zeros_like(out), torch.zeros_like(lse)
        st.attn(tab, n, q, o, k_new=k1, v_new=v1, lse=l)
        assert torch.equal(o, out) and torch.equal(l, lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8", "int4"])
@pytest.mark.parametrize("page,width,append", [(16, 9, True), (16, 9, False), (5, 26, True), (24, 400, True), (5, 2000, False), (64, 200, True)])
def test_what_stands_in_places_that_nobody_needs(fmt, page, width, append):
    """Short and long calls, sequences that are left out and such without rows: numbers of no page, of pages full of NaN or of other sequences'
    pages in the places behind a sequence's rows are as good as -1."""
    lens, h_q, h_kv = [100, -1, 0, page, 17, -5, 127], 8, 2
    st, table, g = cache(fmt, 65, lens, page, h_q, h_kv)
    need = [0 if n < 0 else -(-(n + append) // page) for n in lens]
    at = np.arange(width)[None, :] < np.array(need)[:, None]
    table = np.where(at, np.pad(table, ((0, 0), (0, max(0, width - table.shape[1]))))[:, :width], -1)
    nan = next(i for i in range(st.pages) if i not in table)
    x = torch.full((1, page, h_kv, 128), float("nan"), device=DEV, dtype=torch.bfloat16)
    st.append(ints([[nan]]), x, x)
    q, k1, v1 = rows(g, 7, h_q, 128), rows(g, 7, h_kv, 128), rows(g, 7, h_kv, 128)
    kw = dict(k_new=k1, v_new=v1) if append else {}
    got = []
    for odd in (None, [-2 ** 31, 2 ** 31 - 1, st.pages, nan], [nan, int(table[0, 0])]):
        t = table if odd is None else np.where(at, table, np.array(odd)[np.arange(7 * width).reshape(7, width) % len(odd)])
        out, lse = torch.full_like(q, 7), torch.full((7, h_q), 7.0, device=DEV)
        st.attn(ints(t), ints(lens), q, out, lse=lse, **kw)
        got.append((out, lse, *(x.view(torch.uint8).clone() for x in (st.k, st.v, st.k_scale, st.v_scale) if x is not None)))
    out, lse = got[0][:2]
    assert torch.isfinite(out).all() and (out[[1, 5]] == 7).all() and (lse[[1, 5]] == 7).all() and not (out[[0, 3, 4, 6]] == 7).all(-1).any()
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8", "int4"])
@pytest.mark.parametrize("page,places,interleaved", [(16, 12, False), (5, 36, True), (16, 520, True)])      # short calls, and long ones
def test_every_byte_that_a_captured_step_leaves(fmt, page, places, interleaved):
    """A captured step that rotates, appends and attends, replayed while lengths and tables grow, next to the same calls one by one: all bytes of
    rows and scales of K and V are the same, those that the steps wrote and all others, which are as they were."""
    B, h_q, h_kv, n_pages = 3, 8, 2, 120
    g = gen(66)
    rot = gkv.Rotary(plain(64), interleaved=interleaved, device=DEV)
    st, two = (gkv.PagedStore(fmt, pages=n_pages, page_size=page, h_q=h_q, h_kv=h_kv, max_batch=B, device=DEV) for _ in range(2))
    every = torch.arange(n_pages, dtype=torch.int32, device=DEV)[:, None]
    x = rows(g, 2, n_pages, page, h_kv, 128)
    for s in (st, two):
        s.append(every, x[0], x[1])
    buffers = [[t.view(torch.uint8) for t in (s.k, s.v, s.k_scale, s.v_scale) if t is not None] for s in (st, two)]
    order = np.random.RandomState(4).permutation(n_pages)
    table, length, used = torch.full((B, places), -1, dtype=torch.int32, device=DEV), ints([0, 14, 31]), 0

    def grow():
        nonlocal used
        for b, n in enumerate(length.tolist()):
            for p in range(n // page + 1):
                if table[b, p] < 0:
                    table[b, p] = int(order[used])
                    used += 1

    grow()
    q, k1, v1 = rows(g, B, h_q, 128), rows(g, B, h_kv, 128), rows(g, B, h_kv, 128)
    out, lse = torch.zeros_like(q), torch.zeros(B, h_q, device=DEV)
    for s in (st, two):                                    # not captured: modules are loaded
        s.attn(table, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
    start = [b.clone() for b in buffers[1]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.attn(table, length, q, out, k_new=k1, v_new=v1, rotary=rot, lse=lse)
    written = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
    for _ in range(40):
        q.copy_(rows(g, B, h_q, 128)), k1.copy_(rows(g, B, h_kv, 128)), v1.copy_(rows(g, B, h_kv, 128))
        graph.replay()
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        turned = torch.empty_like(k1)
        rot.apply(length[:, None], k1[:, None], q_out=turned[:, None])
        two.append(table, turned[:, None], v1[:, None], first=length)
        two.attn(table, length + 1, q, o2, rotary=rot, lse=l2)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        for b, n in enumerate(length.tolist()):
            written[int(table[b, n // page]), n % page] = True
        length += 1
        grow()
    for a, b, c in zip(*buffers, start):
        assert torch.equal(a, b)
        assert torch.equal(a.transpose(1, 2)[~written], c.transpose(1, 2)[~written])


# ---------------------------------------------------------------------------------------------- next to a backward pass
class Turn(torch.autograd.Function):
    """The rotation in a model that is trained."""

    @staticmethod
    def forward(ctx, rot, pos, q, k):
        ctx.rot = rot
        ctx.save_for_backward(pos)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        rot.apply(pos, q, k, q_out=qo, k_out=ko)
        return qo, ko

    @staticmethod
    def backward(ctx, dq, dk):
        (pos,) = ctx.saved_tensors
        dq, dk = dq.clone(), dk.clone()
        ctx.rot.apply(pos, dq, dk, transpose=True)
        return None, None, dq, dk


def test_a_rotation_within_a_backward_pass():
    """Gradients of a sum of products of turned q and k, against the same in fp64 by torch. Of q and k that are turned by rounded cos and sin the
    product is off by what the tolerance of a rotation says of its factors; a gradient is one of them, times the weight, turned once more."""
    g = gen(63)
    q, k = (randn(g, "fp32", 2, 9, 3, 80).requires_grad_() for _ in range(2))
    w = randn(g, "fp32", 2, 9, 3, 80)
    pos = torch.randint(0, 3000, (2, 9), generator=g, device=DEV, dtype=torch.int32)
    rot = gkv.Rotary(plain(40), head_dim=80, device=DEV)
    qo, ko = Turn.apply(rot, pos, q, k)
    (qo * ko * w).sum().backward()
    angle = torch.from_numpy(pref.angles(rot.turns.cpu().numpy().view(np.uint64), pos.cpu().numpy())).to(DEV)[:, :, None]
    c, s = torch.cos(angle), torch.sin(angle)

    def turn(x):
        a, b = x[..., :20], x[..., 20:40]
        return torch.cat((a * c - b * s, b * c + a * s, x[..., 40:]), -1)

    q64, k64 = (x.detach().double().requires_grad_() for x in (q, k))
    (turn(q64) * turn(k64) * w.double()).sum().backward()
    # numbers below 6, so a pair's magnitudes add up to less than 12 and a turned one to less than 9: 4 u 12 + u 9 for it, times w below 6, and
    # the product's rounding u 54: 400 u; turned, two of them and 4 u 2 54 + u 77 of its own: 1310 u
    assert all(float(x.detach().abs().max()) < 6 for x in (q, k, w))
    for x, y in ((q, q64), (k, k64)):
        assert (x.grad.double() - y.grad).abs().max() < 1310 * 2.0 ** -24


@pytest.mark.parametrize("which", ["q", "k", "q_out", "k_out"])
def test_a_rotation_that_a_backward_pass_would_not_see_is_refused(which):
    rot = gkv.Rotary(plain(128), device=DEV)
    pos = torch.zeros(1, 2, dtype=torch.int32, device=DEV)
    given = {n: torch.ones(1, 2, 1, 128, device=DEV) for n in ("q", "k", "q_out", "k_out")}
    given[which].requires_grad_()
    with pytest.raises(ValueError, match=f"{which} requires grad"):
        rot.apply(pos, given["q"], given["k"], q_out=given["q_out"], k_out=given["k_out"])
    with torch.no_grad():
        rot.apply(pos, given["q"], given["k"], q_out=given["q_out"], k_out=given["k_out"])
    assert (given["q_out"] == 1).all() and (given["k_out"] == 1).all()


def test_written_tensors_count_as_changed():
    """Every tensor that a call writes: a backward pass that has kept one refuses it, as after torch's own writes. Those that are only read, and
    those of a refused call, do not."""
    g = gen(64)
    rot = gkv.Rotary(plain(128), device=DEV)
    pos, n, tab = torch.zeros(1, 4, dtype=torch.int32, device=DEV), ints([3]), ints([[0]])
    x, y, z, u = (rows(g, 1, 4, 2, 128) for _ in range(4))
    q, out, lse, k1 = rows(g, 1, 2, 128), rows(g, 1, 2, 128), torch.zeros(1, 2, device=DEV), rows(g, 1, 2, 128)
    paged = gkv.PagedStore("int8", pages=1, page_size=16, h_q=2, h_kv=2, max_batch=1, device=DEV)
    flat = gkv.KVStore("int8", batch=1, h_q=2, h_kv=2, capacity=16, device=DEV)
    read = (pos, n, tab, q, k1, x, y)
    for call, written in (
            (lambda: rot.apply(pos, z), [z]), (lambda: rot.apply(pos, z, u), [z, u]), (lambda: rot.apply(pos, x, q_out=z), [z]),
            (lambda: rot.apply(pos, x, z, q_out=u), [u, z]), (lambda: paged.append(tab, x, y), []), (lambda: paged.read(tab, z, u), [z, u]),
            (lambda: paged.attn(tab, n, q, out, k_new=k1, v_new=k1), [out]), (lambda: paged.attn(tab, n, q, out, lse=lse), [out, lse]),
            (lambda: flat.write(x, y), []), (lambda: flat.read(z, u), [z, u]), (lambda: flat.attn(n, q, out, lse=lse), [out, lse])):
        before = {id(t): t._version for t in (*read, z, u, out, lse)}
        call()
        for t in (*read, z, u, out, lse):
            assert (t._version > before[id(t)]) == any(t is w for w in written)
    before = x._version
    with pytest.raises(gkv.GKVError):
        rot.apply(pos, x, y, q_out=x, k_out=x)
    assert x._version == before
    leaf = torch.ones(1, 4, 2, 128, device=DEV, requires_grad=True)
    h = leaf * 2
    loss = (h * h).sum()
    with torch.no_grad():
        rot.apply(pos + 5, h)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    with torch.inference_mode():
        i = torch.ones(1, 4, 2, 128, device=DEV)
    rot.apply(pos + 5, i)                                      # has no count of changes
    assert not (i == 1).all()
