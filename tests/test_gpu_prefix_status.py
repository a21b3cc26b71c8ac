"""An expired wait of the prefix kernel under gkv_decode_attn_prefix: latched, reported once by the poll, and the context goes on after
its state has been declared anew. The kernel is told to take its waits for expired, so that the path is taken for real and nothing
traps, faults or hangs."""
import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
import store_reference as ref
from test_gpu_store import DEV, f64, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,m", [(3, 333), (40, 1500)])      # rows of an item in one tile of 128 and in two; one run and several
def test_an_expired_wait_is_reported_once(B, m):
    gkv.build_library()
    Hq, H, start = 8, 2, 20
    cache = gkv.GKVCache(gkv.make_config(n_layers=1, batch=B, h_q=Hq, h_kv=H, b=48, buffer=24, w=16, s=16, fuse_window_scores=False), DEV)
    g = gen(51)
    k, v = randn(g, B, H, start, 128), randn(g, B, H, start, 128)
    kp, vp = randn(g, 1, H, m, 128), randn(g, 1, H, m, 128)
    prefix, ws = gkv.Prefix(kp, vp, [m]), cache.prefix_workspace(1, m)
    q, kn, vn, out = randn(g, B, Hq, 128), randn(g, B, H, 128), randn(g, B, H, 128), torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=DEV)

    def step():
        cache.k[0, :, :, :start], cache.v[0, :, :, :start] = k, v
        cache.set_state(0, start, 0, 0)
        cache.decode_attn_prefix(0, q, kn, vn, prefix, out, ws)

    def right():
        K, V = torch.cat((k, kn[:, :, None]), 2), torch.cat((v, vn[:, :, None]), 2)
        for b in (0, B - 1):
            for h in range(H):
                hs = slice(4 * h, 4 * h + 4)
                want, _, tol, _ = ref.attend(f64(q[b, hs]), f64(K[b, h]), f64(V[b, h]), f64(kp[0, h]), f64(vp[0, h]), ref.U_BF16)
                if not (np.abs(f64(out[b, hs]) - want) <= tol).all():
                    return False
        return True

    step()
    cache.poll()
    assert right()
    gkv.gkv_selftest_prefix_wait(cache.ctx)
    step()
    with pytest.raises(gkv.GKVError) as e:
        cache.poll()
    assert e.value.status == gkv.GKV_ERR_TIMEOUT
    assert torch.isnan(out).all()
    cache.poll()                                       # reported once
    step()                                             # and taken for expired once
    cache.poll()
    assert right()


@pytest.mark.parametrize("rows", [0, 5])
def test_a_context_with_a_prefix_without_rows_is_an_ordinary_step(rows):
    B, Hq, H = 3, 8, 2
    cache = gkv.GKVCache(gkv.make_config(n_layers=1, batch=B, h_q=Hq, h_kv=H, b=48, buffer=24, w=16, s=16, fuse_window_scores=False), DEV)
    g = gen(52)
    empty = torch.zeros((1, H, rows, 128), dtype=torch.bfloat16, device=DEV)
    prefix, ws = gkv.Prefix(empty, empty, [0]), cache.prefix_workspace(1, 0)
    out = torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=DEV)
    for t in range(20):
        q, kn, vn = randn(g, B, Hq, 128), randn(g, B, H, 128), randn(g, B, H, 128)
        cache.decode_attn_prefix(0, q, kn, vn, prefix, out, ws)
        assert cache.len[0, 0].tolist() == [t + 1] * B and cache.state(0)[0] == t + 1
        assert torch.equal(cache.k[0, :, :, t], kn) and torch.equal(cache.v[0, :, :, t], vn)
        for h in range(H):
            hs = slice(4 * h, 4 * h + 4)
            want, _, tol, _ = ref.attend(f64(q[1, hs]), f64(cache.k[0, 1, h, :t + 1]), f64(cache.v[0, 1, h, :t + 1]), weight_unit=ref.U_BF16)
            assert (np.abs(f64(out[1, hs]) - want) <= tol).all()
    cache.poll()
