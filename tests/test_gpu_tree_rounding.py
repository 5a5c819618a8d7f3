"""Where bf16 rounds the weight of a token, on the GPU: fp8 contexts of several tiles."""
import numpy as np
import pytest
import torch

import gen
import oracle
from tests.tree_cases import TreeRun, check_tree, make

pytestmark = pytest.mark.gpu


def rows_of(w, b, n):
    """K and V of the first head's n tokens and their v_scales, in float64."""
    table, page = oracle.e4m3_table(), lambda t: w.block_table[b, t // w.P]
    scale = lambda s: np.array([s[page(t), 0] for t in range(n)], dtype=np.float64)[:, None]
    codes = lambda pool: np.array([table[pool[page(t), 0, t % w.P]] for t in range(n)])
    return codes(w.k_pool) * scale(w.k_scale), codes(w.v_pool) * scale(w.v_scale), scale(w.v_scale)[:, 0]


@pytest.mark.parametrize("at", [0, 5, 350, 600])
@pytest.mark.parametrize("N,Hq", [(1, 1), (40, 1), (60, 2)])
def test_a_token_that_moves_the_maximum_is_not_rounded(N, Hq, at):
    """The running maximum moves to a logit that exceeds it by more than 8 (log2, v_scale with it): p v_scale is 1 there and has no rounding.  So a row with one
    token more than 2^8 times as weighty as any other carries the output's rounding, 2^-8 of every other share, and what fp32 logits and sums add."""
    n = 700
    w = make("moves", 51, [n], Hq=Hq, Hkv=1, D=64, P=1, kv="fp8_e4m3", pillar_frac=0.0)
    w.k_scale[w.block_table[0, 0]] /= 4                                        # (no sinks)
    w.k_scale[w.block_table[0, 1]] /= 4
    line = gen.f32_from_bf16_bits(gen.bf16_bits_from_f32(np.random.default_rng(3).standard_normal(64).astype(np.float32)))
    w.k_pool[w.block_table[0, at], 0, 0] = np.where(line < 0, 0xc0, 0x40)      # 2.0 in the direction of the queries
    w.k_scale[w.block_table[0, at]] = 0.8
    w.v_scale[w.block_table[0, at]] = np.float32(0.0061)                       # (no power of two)
    q = np.broadcast_to(line, (1, N, Hq, 64)).copy()
    run = TreeRun(w, N, None, [[2 ** (i + 1) - 1 for i in range(N)]],
                  queries_of=(torch.from_numpy(gen.bf16_bits_from_f32(q).view(np.int16)).view(torch.bfloat16), q.astype(np.float64)))
    run.run()
    torch.cuda.synchronize()
    check_tree(run, f"moves {N} {at}")
    k, v, vs = rows_of(w, 0, n)
    x = k @ line.astype(np.float64) * w.sm_scale
    ahead = x / np.log(2) + np.log2(vs)
    assert ahead[at] - np.delete(ahead, at).max() > 8.1                        # (a condition on the inputs)
    prob = 2 * w.D * 2.0 ** -24 * (np.abs(k) @ np.abs(line)).max() * w.sm_scale + (n + 32) * 2.0 ** -24
    got = run.out.double().cpu().numpy()
    for i in range(N):
        seen = n - N + i + 1
        p = np.exp(x[:seen] - x.max())
        p /= p.sum()
        want, size = p @ v[:seen], p @ np.abs(v[:seen])
        rest = size - p[at] * np.abs(v[at])
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * (1 + 2.0 ** -8) * rest + prob * size
        assert (np.abs(got[0, i] - want) <= bound).all(), (i, (np.abs(got[0, i] - want) / bound).max())


@pytest.mark.parametrize("N,Hq", [(1, 1), (40, 1), (60, 2)])
def test_a_maximum_that_grows_by_less(N, Hq):
    """Logits that climb by less than 8 from tile to tile leave the maximum where the first tile set it: every share is rounded, by 2^-8 of itself at the most."""
    n = 700
    w = make("climbs", 52, [n], Hq=Hq, Hkv=1, D=64, P=1, kv="fp8_e4m3", pillar_frac=0.0)
    line = gen.f32_from_bf16_bits(gen.bf16_bits_from_f32(np.random.default_rng(4).standard_normal(64).astype(np.float32)))
    w.k_pool[w.block_table[0], 0, 0] = np.where(line < 0, 0xb8, 0x38)          # 1.0 in the direction of the queries
    w.k_scale[w.block_table[0], 0] = np.linspace(0.0, 7.5 * np.log(2) / (np.abs(line).sum() * w.sm_scale), n)
    q = np.broadcast_to(line, (1, N, Hq, 64)).copy()
    run = TreeRun(w, N, None, [[2 ** (i + 1) - 1 for i in range(N)]],
                  queries_of=(torch.from_numpy(gen.bf16_bits_from_f32(q).view(np.int16)).view(torch.bfloat16), q.astype(np.float64)))
    run.run()
    torch.cuda.synchronize()
    check_tree(run, f"climbs {N}")
