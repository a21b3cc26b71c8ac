"""Rotations and caches in pages on the GPU at the ends of what their description allows."""
import numpy as np
import pytest
import torch

import paper_2512_00504_b200 as gkv
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
