"""Rotary positions on the GPU against the fp64 reference: both orders of pairs, parts of the head, all types, every width of access,
strides, ragged counts, far and negative positions, and the transposed rotation as the gradient."""
import math

import numpy as np
import pytest
import torch

import pages_reference as pref
import paper_2512_00504_b200 as gkv

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def built():
    gkv.build_library()
    gkv.build_binding()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, dtype, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(TYPES[dtype])


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def plain(rot):
    return [10000.0 ** (-2 * i / rot) for i in range(rot // 2)]


def check(rot, dtype, pos, x, y, transpose=False):
    turns = rot.turns.cpu().numpy().view(np.uint64)
    want, mag = pref.rotate(f64(x), pref.angles(turns, pos.cpu().numpy()), rot.desc.interleaved, rot.desc.factor, transpose)
    off = np.abs(f64(y) - want)
    assert (off <= pref.rotation_tolerance(want, mag, dtype)).all(), off.max()


# head, rot: every width of access of each type (8, 4, 2 and 1 pairs), runs that do not divide a block's threads, none to copy
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head,part", [(128, 128), (128, 64), (64, 32), (80, 80), (80, 40), (80, 20), (96, 48), (6, 2), (10, 10), (256, 256), (512, 512), (512, 2)])
def test_pairs_and_widths(dtype, interleaved, head, part):
    g = gen(head + part)
    q, k = randn(g, dtype, 3, 5, 4, head), randn(g, dtype, 3, 5, 2, head)
    pos = torch.randint(0, 5000, (3, 5), generator=g, device=DEV, dtype=torch.int32)
    rot = gkv.Rotary(plain(part), head_dim=head, interleaved=interleaved, factor=1.25 if part == 64 else 1.0, device=DEV)
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    q0, k0 = q.clone(), k.clone()
    rot.apply(pos, q, k, q_out=qo, k_out=ko)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    check(rot, dtype, pos, q, qo)
    check(rot, dtype, pos, k, ko)
    rot.apply(pos, q, k)                       # in place: the same bits
    assert torch.equal(q, qo) and torch.equal(k, ko)
    rot.apply(pos, q0, q_out=(alone := torch.zeros_like(q0)))
    assert torch.equal(alone, qo)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_slices_of_a_projection_at_any_alignment(dtype, interleaved):
    """q and k within one tensor whose rows begin anywhere, written to another with a layout of its own; what lies between stays."""
    g = gen(5)
    for shift in (0, 1, 2, 4):
        flat = randn(g, dtype, 2 * 7 * 9 * 96 + 64)
        qkv = flat[shift:shift + 2 * 7 * 9 * 96].view(2, 7, 9, 96)
        q, k = qkv[:, :, :5], qkv[:, :, 5:7]
        wide = torch.full((2, 9, 7, 100), 3.0, device=DEV, dtype=TYPES[dtype])      # [batch][heads][tokens]
        qo, ko = wide[:, :5, :, :96].transpose(1, 2), wide[:, 6:8, :, 4:].transpose(1, 2)
        pos = torch.randint(0, 99, (2, 7), generator=g, device=DEV, dtype=torch.int32)
        rot = gkv.Rotary(plain(48), head_dim=96, interleaved=interleaved, device=DEV)
        rot.apply(pos, q, k, q_out=qo, k_out=ko)
        check(rot, dtype, pos, q, qo)
        check(rot, dtype, pos, k, ko)
        left = wide.clone()
        left[:, :5, :, :96] = 3.0
        left[:, 6:8, :, 4:] = 3.0
        assert (left == 3.0).all()


@pytest.mark.parametrize("batch,tokens,h_q,h_k", [(1, 1, 1, 1), (1, 1, 28, 4), (64, 1, 64, 8), (1, 1023, 28, 4), (3, 700, 64, 8), (700, 3, 5, 1), (2, 2049, 1, 1)])
def test_batches_and_lengths(batch, tokens, h_q, h_k):
    g = gen(batch + tokens)
    q, k = randn(g, "bf16", batch, tokens, h_q, 128), randn(g, "bf16", batch, tokens, h_k, 128)
    pos = torch.arange(tokens, device=DEV, dtype=torch.int32) + torch.randint(0, 100000, (batch, 1), generator=g, device=DEV, dtype=torch.int32)
    rot = gkv.Rotary.scaled(1e6, scaling="yarn", scale=4, original=32768, device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    rot.apply(pos, q, k, q_out=qo, k_out=ko)
    check(rot, "bf16", pos, q, qo)
    check(rot, "bf16", pos, k, ko)


def test_counts_leave_the_rest_as_it_was():
    g = gen(8)
    q, k = randn(g, "bf16", 6, 33, 4, 128), randn(g, "bf16", 6, 33, 2, 128)
    q[:, 32] = math.nan                        # never looked at
    q0 = q.clone()
    pos = torch.arange(33, device=DEV, dtype=torch.int32).expand(6, 33)      # one row of positions for all
    count = [32, 0, -5, 1, 17, 9]
    rot = gkv.Rotary(plain(128), device=DEV)
    qo, ko = torch.full_like(q, 2.5), torch.full_like(k, 2.5)
    rot.apply(pos, q, k, q_out=qo, k_out=ko, count=ints(count))
    for b, n in enumerate(count):
        n = max(n, 0)
        if n:
            check(rot, "bf16", pos[b:b + 1, :n], q[b:b + 1, :n], qo[b:b + 1, :n])
            check(rot, "bf16", pos[b:b + 1, :n], k[b:b + 1, :n], ko[b:b + 1, :n])
        assert (qo[b, n:] == 2.5).all() and (ko[b, n:] == 2.5).all()
    rot.apply(pos, q, count=ints([99] * 6))
    check(rot, "bf16", pos[:, :32], q0[:, :32], q[:, :32])
    rot.apply(pos[:, :0], q[:, :0])            # no tokens


def test_far_and_negative_positions():
    """Angles are exact to a turn at any position: against fractions of a turn in whole numbers, and near ones against fp64."""
    g = gen(9)
    pos = ints([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1234567890, -987654321, 1 << 20, 131071]])
    x = randn(g, "fp32", 1, 9, 3, 128)
    for rot in (gkv.Rotary(plain(128), device=DEV), gkv.Rotary([0.0, 1e-9, 1.0, 2 * math.pi, 3.0, 1e4], device=DEV)):
        y = torch.empty_like(x)
        rot.apply(pos, x, q_out=y)
        check(rot, "fp32", pos, x, y)
    rot = gkv.Rotary(plain(128), device=DEV)
    rot.apply(pos, x, q_out=y)
    near = [0, 1, 2, 7, 8]
    angle = pos.cpu().numpy()[:, near, None].astype(np.float64) * np.array(plain(128))
    want, mag = pref.rotate(f64(x[:, near]), angle, False)
    # fp64's product and argument: 2^20 turns at most, 2^-52 of it, which is 2^-32 next to the 2^-22 of the kernel's own
    assert (np.abs(f64(y[:, near]) - want) <= pref.rotation_tolerance(want, mag * 1.001, "fp32")).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_transposed_rotation_is_the_gradient(interleaved):
    g = gen(10)
    x, dy = randn(g, "fp32", 2, 9, 3, 80), randn(g, "fp32", 2, 9, 3, 80)
    pos = torch.randint(-3000, 3000, (2, 9), generator=g, device=DEV, dtype=torch.int32)
    rot = gkv.Rotary(plain(40), head_dim=80, interleaved=interleaved, factor=1.5, device=DEV)
    dx = torch.empty_like(x)
    rot.apply(pos, dy, q_out=dx, transpose=True)
    check(rot, "fp32", pos, dy, dx, transpose=True)
    # against differences of sum(y * dy): the rotation is linear, so a step of 1 along e is the derivative up to roundings. y and y' are
    # off by 5 u (|a| + |b|) 1.5 each, with |a|, |b| < 8 (normal numbers and a step of 1): 240 u; two elements of dy (< 8) take part
    for e in (0, 1, 19, 20, 39, 40, 79):
        y0, y1, x1 = torch.empty_like(x), torch.empty_like(x), x.clone()
        x1[..., e] += 1.0
        rot.apply(pos, x, q_out=y0)
        rot.apply(pos, x1, q_out=y1)
        slope = ((y1.double() - y0.double()) * dy.double()).sum(-1) / (x1.double() - x.double())[..., e]
        assert (slope - dx[..., e].double()).abs().max() < 240 * 2.0 ** -24 * 2 * 8 * 2
    # bf16 gradients of a step as autograd would hand them back
    back = randn(g, "bf16", 2, 9, 3, 80)
    dxb = torch.empty_like(back)
    rot.apply(pos, back, q_out=dxb, transpose=True)
    check(rot, "bf16", pos, back, dxb, transpose=True)


def test_nan_and_infinity_stay_in_their_pair():
    x = torch.ones(1, 1, 1, 128, device=DEV)
    x[..., 3], x[..., 40], x[..., 127] = math.nan, math.inf, -math.inf
    rot = gkv.Rotary(plain(64), device=DEV)
    y = torch.empty_like(x)
    rot.apply(ints([[5]]), x, q_out=y)
    fine = torch.ones(128, dtype=torch.bool)
    fine[[3, 35, 8, 40, 127]] = False
    assert torch.isfinite(y[0, 0, 0].cpu())[fine].all() and torch.isnan(y[..., [3, 35]]).all() and not torch.isfinite(y[..., [8, 40]]).any()
    assert y[0, 0, 0, 127] == -math.inf


def test_keys_kept_by_an_eviction_move_to_their_places_in_the_cache():
    """Rows of a compressed cache turned from their own positions to their places: by the difference, through views of the cache."""
    cfg = gkv.make_config(n_layers=1, batch=2, h_q=8, h_kv=2, b=64, buffer=32, w=8, s=32, fuse_window_scores=False, track_positions=True)
    cache = gkv.GKVCache(cfg, DEV)
    g = gen(11)
    cache.k.copy_(randn(g, "bf16", *cache.k.shape))
    cache.v.copy_(randn(g, "bf16", *cache.v.shape))
    cache.pos.copy_(torch.arange(96, device=DEV, dtype=torch.int32).expand_as(cache.pos))
    cache.set_state(-1, 96, 0, 32)
    cache.evict(-1, q_window=randn(g, "bf16", 1, 2, 8, 8, 128))
    heads, kept = cache.k.view(4, 1, 96, 128).transpose(1, 2)[:, :64], cache.pos.view(4, 96)[:, :64]      # a head as a sequence
    before = heads.clone()
    shift = torch.arange(64, device=DEV, dtype=torch.int32) - kept
    assert int(shift.min()) < 0
    rot = gkv.Rotary(plain(128), device=DEV)
    rot.apply(shift, heads)
    check(rot, "bf16", shift, before, heads)


def test_another_stream_and_a_captured_graph():
    g = gen(12)
    x = randn(g, "bf16", 4, 300, 8, 128)
    pos = torch.arange(300, device=DEV, dtype=torch.int32).expand(4, 300).contiguous()
    rot = gkv.Rotary(plain(128), device=DEV)
    want = torch.empty_like(x)
    rot.apply(pos, x, q_out=want)
    torch.cuda.synchronize()
    s, got = torch.cuda.Stream(), torch.zeros_like(x)
    with torch.cuda.stream(s):
        rot.apply(pos, x, q_out=got)
    s.synchronize()
    assert torch.equal(got, want)
    graph, got = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    with torch.cuda.graph(graph):
        rot.apply(pos, x, q_out=got)
    pos += 77                                   # the replay reads the positions as they are then
    rot.apply(pos, x, q_out=want)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_tensors_that_are_refused():
    rot = gkv.Rotary(plain(128), device=DEV)
    x, pos = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    for args, kw in (((pos, x.double()), {}), ((pos.long(), x), {}), ((pos[:1], x), {}), ((pos[:, :2], x), {}), ((pos, x[0]), {}), ((pos, x[..., :64]), {}),
                     ((pos, x.cpu()), {}), ((pos.cpu(), x), {}), ((pos, x, x.float()), {}), ((pos, x, x[:1]), {}), ((pos, x, x[:, :2]), {}), ((pos, x), dict(k_out=x)),
                     ((pos, x), dict(q_out=x[:1])), ((pos, x), dict(q_out=x.float())), ((pos, x), dict(count=pos[:, 0].long())), ((pos, x), dict(count=pos[0])),
                     ((pos, x.transpose(2, 3)), {}), ((pos, [1]), {}), ((None, x), {})):
        with pytest.raises(ValueError):
            rot.apply(*args, **kw)
    for args, kw in (((pos, x), dict(q_out=x[:, :, :1].expand(2, 3, 4, 128))), ((pos, x, x.clone()), dict(q_out=x, k_out=x))):
        with pytest.raises(gkv.GKVError):
            rot.apply(*args, **kw)
