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


@pytest.mark.parametrize("kv,flags", TYPES)
@pytest.mark.parametrize("Hq,N", [(4, 8), (4, 12), (4, 30), (8, 40)])
def test_keys_that_one_node_sees(kv, flags, Hq, N):
    """K of the last two nodes, each seen by itself only, infinite in one dimension, then finite and large: nobody else's logits have them, so nobody
    else's running maximum moves.  (A page of one token each: an fp8 row is made large by its scale.)"""
    lens, q = [N + 3, 300, 1500], "f32" if kv == "f32" else "bf16"
    rng = np.random.default_rng(N)
    w = make("keys", 32, lens, Hq=Hq, Hkv=1, D=64, P=1, kv=kv, q=q)
    words = alone([ancestors(rng, N) for _ in lens], [N - 2, N - 1])
    clean = TreeRun(w, N, None, words, seed=N, flags=flags)
    clean.run()
    torch.cuda.synchronize()
    for what in ("large",) if kv == "fp8_e4m3" else ("inf", "large"):
        print(f"[case] {what} Hq={Hq} N={N} {kv} flags={flags}", flush=True)
        k, scale = w.k_pool.copy(), None if w.k_scale is None else w.k_scale.copy()
        for b, n in enumerate(lens):
            for t in (n - 2, n - 1):
                if what == "inf":
                    set_row(w, w.k_pool, b, t, STORED[kv]["inf"], 5)
                elif kv == "fp8_e4m3":
                    w.k_scale[w.block_table[b, t]] *= 1024
                elif kv == "bf16":
                    w.k_pool[w.block_table[b, t]] += np.uint16(10 << 7)            # the exponent
                else:
                    w.k_pool[w.block_table[b, t]] *= 1024
        dirty = TreeRun(w, N, None, words, seed=N, flags=flags)
        dirty.run()
        torch.cuda.synchronize()
        w.k_pool, w.k_scale = k, scale
        assert torch.equal(dirty.out[:, :N - 2], clean.out[:, :N - 2]), what
        assert torch.equal(dirty.lse[:, :N - 2], clean.lse[:, :N - 2]), what
        assert not torch.equal(dirty.lse[:, N - 2:], clean.lse[:, N - 2:])
