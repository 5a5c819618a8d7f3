"""Rotary positions and appends at the ends of what they take, on the GPU."""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_01278_amd as pa
from tests.test_gpu_rotate import Append
from tests.tree_cases import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("P", [16, 64])                   # (rows kept in registers, and read twice)
@pytest.mark.parametrize("scale", [2.0 ** -149, 2.0 ** -130, 2.0 ** -127, 2.0 ** -110, 2.0 ** -100, 2.0 ** -99, 2.0 ** -98, 0.0])
@pytest.mark.parametrize("fill", [0.0, 1e-30, 2.0 ** -91])
def test_older_tokens_next_to_nothing(P, scale, fill):
    """The page's scale is theirs, their codes stay, and new tokens of nothing are zeros (from 2^-90 / 448 on, what the scale holds)."""
    w = make("tiny", 21, [P + 12, 9], Hq=2, Hkv=2, D=64, P=P, kv="fp8_e4m3", q="f32")
    w.k_scale[:], w.v_scale[:] = scale, scale
    a = Append(w, [4, 3], fused=False)
    a.k[:], a.v[:] = fill, -fill
    a.rows = torch.cat([a.q, a.k, a.v], dim=1).cpu()
    a.run()
    a.check()
    for pool, at, was in ((a.kv.k_pool, a.kv.k_scale, w.k_pool), (a.kv.v_pool, a.kv.v_scale, w.v_pool)):
        for b, first, end in ((0, 8, 12), (1, 6, 9)):
            page = w.block_table[b, 1 if b == 0 else 0]
            assert (at[page] == scale).all() and np.array_equal(pool[page, :, :first].cpu().numpy(), was[page, :, :first])
            new = oracle.e4m3_table()[pool[page, :, first:end].cpu().numpy()]
            assert (np.abs(new * scale) <= 2.0 ** -90).all() and np.isfinite(new).all()
            if scale < 2.0 ** -90 / 448:
                assert (new == 0).all()
