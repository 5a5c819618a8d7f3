"""What a node of a tree does not see, on the GPU: whatever the cache holds there, the node's results are those without it, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from tests.tree_cases import TreeRun, ancestors, make

pytestmark = pytest.mark.gpu

GENERIC = pa.PILLAR_FLAG_GENERIC_KERNELS
TYPES = [("bf16", 0), ("fp8_e4m3", 0), ("f32", 0), ("bf16", GENERIC)]
STORED = {"f32": dict(inf=np.float32(np.inf), nan=np.float32(np.nan)), "bf16": dict(inf=np.uint16(0x7f80), nan=np.uint16(0xffc0)),
          "fp8_e4m3": dict(inf=np.uint8(0x7f), nan=np.uint8(0xff))}            # (e4m3 has no infinities)


def alone(words, nodes):
    """The same trees, in which each of `nodes` is seen by itself only."""
    mask = sum(1 << j for j in nodes)
    return [[word & ~mask | (1 << i if i in nodes else 0) for i, word in enumerate(row)] for row in words]


def set_row(w, pool, b, t, value, dims=slice(None)):
    pool[w.block_table[b, t // w.P], :, t % w.P, dims] = value


@pytest.mark.parametrize("kv,flags", TYPES)
@pytest.mark.parametrize("N,hit", [(32, [31]), (33, [31]), (40, [30, 31, 32]), (64, [31]), (64, [0, 31, 32, 63])])
def test_nodes_at_the_ends_of_the_words(kv, flags, N, hit):
    """V of nodes 31, 32 and 63: the bits at the ends of the two halves of a node's word.  Block tables say -1 for what is past a context."""
    lens, q = [N, N + 50, 200, 2500 + N], "f32" if kv == "f32" else "bf16"
    rng = np.random.default_rng(N)
    w = make("ends", 31, lens, Hq=4, Hkv=1, D=64, kv=kv, q=q, extra_table_cols=8)
    words = alone([ancestors(rng, N) for _ in lens], hit)
    print(f"[case] N={N} nodes={hit} {kv} flags={flags}", flush=True)
    clean = TreeRun(w, N, None, words, seed=N, flags=flags)
    clean.run()
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for j in hit:
            set_row(w, w.v_pool, b, n - N + j, STORED[kv]["inf" if j % 2 else "nan"], slice(None, None, 3))
    dirty = TreeRun(w, N, None, words, seed=N, flags=flags)
    dirty.run()
    torch.cuda.synchronize()
    others = [i for i in range(N) if i not in hit]
    assert torch.equal(dirty.out[:, others], clean.out[:, others])
    assert torch.equal(dirty.lse, clean.lse) and torch.equal(dirty.scores.nan_to_num(-1), clean.scores.nan_to_num(-1))
    for j in hit:
        seen = dirty.out[:, j].float()
        assert not torch.isfinite(seen[..., ::3]).any()
        for dim in (1, 2):
            assert torch.equal(seen[..., dim::3], clean.out[:, j].float()[..., dim::3])
