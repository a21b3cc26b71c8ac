"""Key/value stores at the ends of their documented range: tokens and rows at the ends of 32 bits."""
import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
import store_reference as ref
from test_gpu_store import DEV, FORMATS, expect_codes, f64, gen, ints, randn, raw

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
