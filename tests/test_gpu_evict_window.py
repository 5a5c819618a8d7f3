"""Sinks and a recent window after an eviction, on the GPU: slots say nothing about age, positions do."""
import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2512_01278_amd as pa
from tests.harness import check_out
from tests.test_gpu_evict import State
from tests.tree_cases import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_a_window_by_positions(kv):
    """A draft over the first 4 and the last 20 tokens of the text, of a cache that keeps 90 of 300 and of 70."""
    B, Hkv, Hq, sink, recent, budgets = 2, 2, 8, 4, 20, [90, 50]
    w = make("window", 71, [300, 70], Hq=Hq, Hkv=Hkv, kv=kv)
    s = State(w, 15)
    dev = s.kv.k_pool.device
    put, ints = lambda x: torch.from_numpy(x).to(dev), lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    weights, positions, now = put(s.weights), put(s.positions), ints([0, 0])
    ws = torch.empty(pa.pillar_evict_workspace_bytes(s.kv), dtype=torch.uint8, device=dev)
    pa.pillar_evict_kv(s.kv, put(s.scores), 1.0, ints([0, 0]), ints(budgets), sink, recent, weights, positions, now, ws)
    assert now.tolist() == budgets
    n = sink + recent
    lists, counts = torch.full((B, Hkv, n), -1, dtype=torch.int32, device=dev), ints([n, n])
    for b in range(B):
        held = positions[b, :, :budgets[b]]
        named = (held < sink) | (held > held.amax(dim=1, keepdim=True) - recent)
        assert named.sum(dim=1).tolist() == [n] * Hkv
        lists[b] = named.nonzero()[:, 1].view(Hkv, n).to(torch.int32)
    by_slot, other = torch.zeros_like(lists), torch.zeros_like(counts)
    pa.pillar_window_indices(now, ints([n, n]), Hkv, sink, n, by_slot, other)
    assert not torch.equal(by_slot, lists)                                     # those are the first and the last slots
    w.q_draft = gen.bf16_bits_from_f32(np.random.default_rng(1).standard_normal((B, Hq, 128), dtype=np.float32))
    q = torch.from_numpy(w.q_draft.view(np.int16)).view(torch.bfloat16).to(dev)
    out = torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device=dev)
    pa.pillar_sparse_decode(s.kv, q, lists, counts, n, out, None, torch.empty(pa.pillar_workspace_bytes(s.kv, 0, n), dtype=torch.uint8, device=dev))
    torch.cuda.synchronize()
    if kv == "fp8_e4m3":
        # (a row that moved was rounded anew, by up to 2^-4 of its values: the reference is the draft on the cache that the eviction leaves)
        r = oracle.evict_kv(w, s.scores, 1.0, [0, 0], budgets, sink, recent, s.weights, s.positions)
        w.k_pool, w.v_pool, w.k_scale, w.v_scale = (r[name] for name in ("k_pool", "v_pool", "k_scale", "v_scale"))
        want = lists.cpu().numpy()
    else:
        # on the cache as it was, where a token's slot is its place
        want = np.array([[list(range(sink)) + list(range(L - recent, L))] * Hkv for L in (300, 70)], dtype=np.int32)
    check_out(out.double().cpu().numpy(), oracle.sparse_decode(w, want, np.array([n, n], dtype=np.int32))[0], w.kv_dtype, "window")
