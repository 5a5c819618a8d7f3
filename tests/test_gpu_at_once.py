"""Calls of two streams at once, on the GPU: each with tensors and a workspace of its own, outputs cleared before every turn."""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_01278_amd as pa
from tests.test_gpu_evict import State
from tests.test_gpu_tree import check_cache
from tests.tree_cases import TreeRun, ancestors, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("N", [3, 9, 40])
def test_two_verifications(kv, N):
    lens = [2900, 300, N + 31]
    runs = [TreeRun(make("at once", s, lens, kv=kv), N, None, [ancestors(np.random.default_rng(b), N) for b in range(3)], seed=s) for s in (1, 2)]
    for r in runs:
        r.run()
    torch.cuda.synchronize()
    outputs = lambda r: (r.out, r.lse, r.scores)
    first = [[t.clone() for t in outputs(r)] for r in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(5):
        for r in runs:
            for t in outputs(r):
                t.fill_(float("nan"))
            r.workspace.fill_(turn)
        torch.cuda.synchronize()
        for r, s in zip(runs, streams):
            r.run(stream=s)
        torch.cuda.synchronize()
        for r, f in zip(runs, first):
            assert all(torch.equal(t.nan_to_num(-1), was.nan_to_num(-1)) for t, was in zip(outputs(r), f)), turn


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("n", [300, 9000])
def test_two_evictions(kv, n):
    """300: rows move in the launch that selects; 9000: in one of their own."""
    states = [State(make("at once", s, [n, n // 3], Hq=4, Hkv=2, D=64, kv=kv), s) for s in (3, 4)]
    dev = states[0].kv.k_pool.device
    put, ints = lambda x: torch.from_numpy(x).to(dev), lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    old, budgets = [n - 9, n // 3], [n // 2, n // 4]
    calls = []
    for s in states:
        cache = [t for t in (s.kv.k_pool, s.kv.v_pool, s.kv.k_scale, s.kv.v_scale) if t is not None]
        calls.append(dict(s=s, cache=cache, was=[t.clone() for t in cache], scores=put(s.scores), old=ints(old), budgets=ints(budgets),
                          ws=torch.empty(pa.pillar_evict_workspace_bytes(s.kv), dtype=torch.uint8, device=dev),
                          want=oracle.evict_kv(s.w, s.scores, 0.75, old, budgets, 2, 10, s.weights, s.positions)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        for c in calls:
            for t, was in zip(c["cache"], c["was"]):
                t.copy_(was)
            c.update(weights=put(c["s"].weights), positions=put(c["s"].positions), now=ints([-7, -7]))
            c["ws"].fill_(turn)
        torch.cuda.synchronize()
        for c, stream in zip(calls, streams):
            pa.pillar_evict_kv(c["s"].kv, c["scores"], 0.75, c["old"], c["budgets"], 2, 10, c["weights"], c["positions"], c["now"], c["ws"], stream=stream)
        torch.cuda.synchronize()
        for c in calls:
            assert c["now"].tolist() == c["want"]["new_lens"].tolist()
            assert np.array_equal(c["positions"].cpu().numpy(), c["want"]["positions"])
            assert np.array_equal(c["weights"].cpu().numpy().view(np.uint32), c["want"]["weights"].view(np.uint32))
            check_cache(c["s"].kv, c["want"])
