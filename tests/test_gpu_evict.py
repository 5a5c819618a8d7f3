"""The bounded cache on the GPU against the oracle, bit for bit; and a serving loop of verification, commit, eviction and draft."""
import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2512_01278_amd as pa
from tests.harness import check_out
from tests.test_gpu_tree import check_cache
from tests.tree_cases import TreeRun, ancestors, cache_of, check_tree, make

pytestmark = pytest.mark.gpu


class State:
    def __init__(self, w, seed, spread=1.0, few=False):
        rng = np.random.default_rng(seed)
        self.w, self.kv = w, cache_of(w)
        n = self.kv.max_seq_len + 5
        shape = (w.B, w.Hkv, n)
        self.scores = rng.random(shape, dtype=np.float32) ** 4
        self.weights = rng.random(shape, dtype=np.float32) * np.float32(spread)
        if few:                                              # many equal weights
            self.scores, self.weights = np.round(self.scores * 3) / np.float32(4), np.round(self.weights * 2)
        self.positions = np.stack([np.stack([rng.permutation(3 * n)[:n] for _ in range(w.Hkv)]) for _ in range(w.B)]).astype(np.int32)

    def check(self, old, budgets, sink, recent, decay=0.75, with_scores=True, alias=None, what=""):
        print(f"[case] {what}: lens={self.w.seq_lens.tolist()[:6]} old={list(old)[:6]} budgets={list(budgets)[:6]} sink={sink} recent={recent}", flush=True)
        dev = self.kv.k_pool.device
        want = oracle.evict_kv(self.w, self.scores if with_scores else None, decay, old, budgets, sink, recent, self.weights, self.positions)
        put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
        ints = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device=dev)
        old_d, bud_d, weights, positions = ints(old), ints(budgets), put(self.weights), put(self.positions)
        now = {None: torch.full((self.w.B,), -7, dtype=torch.int32, device=dev), "old": old_d, "budgets": bud_d, "lens": self.kv.seq_lens}[alias]
        ws = torch.empty(pa.pillar_evict_workspace_bytes(self.kv), dtype=torch.uint8, device=dev)
        pa.pillar_evict_kv(self.kv, put(self.scores) if with_scores else None, decay, old_d, bud_d, sink, recent, weights, positions, now, ws)
        torch.cuda.synchronize()
        assert now.tolist() == want["new_lens"].tolist(), what
        assert np.array_equal(positions.cpu().numpy(), want["positions"]), what
        assert np.array_equal(weights.cpu().numpy().view(np.uint32), want["weights"].view(np.uint32)), what
        check_cache(self.kv, want)


@pytest.mark.parametrize("kv,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64), ("fp8_e4m3", 128), ("fp8_e4m3", 64)])
@pytest.mark.parametrize("P", [1, 16, 64])
def test_eviction(kv, D, P):
    w = make("evict", P, [1, 40, 41, 300, 77, 256, 0], kv=kv, q="f32" if kv == "f32" else "bf16", D=D, P=P, Hq=4, Hkv=2)
    State(w, P).check([0, 30, 41, 290, 0, 255, 0], [5, 30, 20, 200, 64, 0, 3], 2, 4, what="ragged")


@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("sink,recent", [(0, 0), (4, 0), (0, 8), (3, 1000), (100000, 0)])
def test_protected_tokens_and_ties(sink, recent, few):
    w = make("protect", 3, [130, 64, 500, 33], Hq=2, Hkv=2, D=64)
    State(w, 7, few=few).check([100, 64, 480, 0], [50, 20, 490, 32], sink, recent, what="protected")


def test_what_is_not_over_its_budget_stays():
    w = make("stays", 3, [130, 64], Hq=2, Hkv=2, D=64)
    State(w, 8).check([100, 64], [130, 1000], 4, 4, what="room")
    State(w, 8).check([100, 70], [-5, 0], 4, 4, what="none")


def test_without_scores():
    w = make("scoreless", 3, [130, 64], Hq=2, Hkv=2, D=64)
    State(w, 9).check([100, 60], [90, 30], 1, 2, with_scores=False, what="no scores")


@pytest.mark.parametrize("alias", ["old", "budgets", "lens"])
def test_new_lengths_in_place(alias):
    w = make("alias", 3, [130, 64, 200], Hq=4, Hkv=4, D=64)
    State(w, 10).check([100, 60, 200], [90, 30, 77], 1, 2, alias=alias, what=alias)


def test_weights_that_are_no_weights():
    """Infinite ones come first, negative ones and NaN count as 0; denormals keep their order."""
    w = make("odd", 3, [64], Hq=1, Hkv=1, D=64)
    s = State(w, 11)
    s.weights[0, 0, :8] = [np.inf, -1, np.nan, 1e-42, 2e-42, 0, -0.0, 3e38]
    s.scores[:] = 0
    s.weights[0, 0, 8:] = 0
    s.check([64], [5], 0, 0, decay=1.0, what="odd")


@pytest.mark.parametrize("n,keep", [(1023, 600), (1024, 1), (1025, 1024), (4097, 4000), (9000, 1000), (33000, 16500), (70001, 300)])
def test_lengths(n, keep):
    w = make("long", 3, [n], Hq=1, Hkv=1, D=64, kv="bf16")
    State(w, n, spread=3.0).check([n // 2], [keep], 4, 64, what=f"{n}")
    State(w, n, few=True).check([n // 2], [keep], 4, 64, what=f"{n} ties")


@pytest.mark.parametrize("alias", [None, "old", "budgets", "lens"])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_many_requests(kv, alias):
    """More (request, KV head) pairs than compute units: rows move in the launch that selects, unless the new lengths replace what it reads."""
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 200, size=90)
    w = make("many", 3, lens, Hq=4, Hkv=4, D=64, kv=kv)
    State(w, 13).check(rng.integers(0, 200, size=90), rng.integers(0, 150, size=90), 2, 5, alias=alias, what="many")


@pytest.mark.parametrize("n,keep", [(3000, 2990), (9000, 5000), (33000, 32000)])
@pytest.mark.parametrize("P", [1, 32, 256])
def test_long_rows_of_fp8(n, keep, P):
    w = make("long8", 3, [n, n // 3], Hq=1, Hkv=1, D=64, kv="fp8_e4m3", P=P)
    State(w, n).check([n // 2, 0], [keep, n // 7], 4, 64, what=f"{n} P={P}")


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_a_page_of_both_kinds(kv):
    """Slot K' inside a page: its rows below K' receive, its rows beyond are sent, and both go by the scale it had."""
    for keep in range(49, 65):
        w = make("edge", keep, [80], kv=kv, Hq=2, Hkv=2)
        State(w, keep).check([0], [keep], 0, 3, what=f"edge {keep}")


def test_a_request_that_is_replayed():
    w = make("replay", 3, [300, 90], Hq=4, Hkv=2)
    s = State(w, 14)
    dev = s.kv.k_pool.device
    put = lambda x: torch.from_numpy(x).to(dev)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    weights, positions, scores, now = put(s.weights), put(s.positions), put(s.scores), ints([0, 0])
    old, budgets = ints([250, 80]), ints([200, 60])
    ws = torch.empty(pa.pillar_evict_workspace_bytes(s.kv), dtype=torch.uint8, device=dev)
    want = oracle.evict_kv(w, s.scores, 0.75, [250, 80], [200, 60], 2, 10, s.weights, s.positions)
    before = [t.clone() for t in (s.kv.k_pool, s.kv.v_pool, weights, positions)]
    call = lambda: pa.pillar_evict_kv(s.kv, scores, 0.75, old, budgets, 2, 10, weights, positions, now, ws)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        for t, was in zip((s.kv.k_pool, s.kv.v_pool, weights, positions), before):
            t.copy_(was)
        ws.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(positions.cpu().numpy(), want["positions"]) and np.array_equal(weights.cpu().numpy(), want["weights"])
        check_cache(s.kv, want)


@pytest.mark.parametrize("kv,Hq", [("bf16", 8), ("fp8_e4m3", 16)])
def test_a_serving_loop(kv, Hq):
    """Verify a tree, commit a path, evict what the budget does not hold, draft from what is left: three rounds, each against the oracle on the
    cache that the round before left."""
    rng = np.random.default_rng(5)
    N, budget, Hkv, top = 10, 96, 2, 160
    lens = np.array([130, 75, 110])
    w = make("loop", 6, [top] * 3, kv=kv, Hq=Hq, Hkv=Hkv)
    w.seq_lens[:] = lens
    kvc = cache_of(w)
    kvc.max_seq_len = top
    dev = kvc.k_pool.device
    ints = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device=dev)
    weights, positions = torch.zeros(3, Hkv, top, device=dev), torch.zeros(3, Hkv, top, dtype=torch.int32, device=dev)
    old, after = ints([0, 0, 0]), ints([0, 0, 0])
    ws = torch.empty(max(pa.pillar_tree_workspace_bytes(kvc, N), pa.pillar_evict_workspace_bytes(kvc), pa.pillar_workspace_bytes(kvc, 0, budget)),
                     dtype=torch.uint8, device=dev)
    host = lambda t: t.cpu().numpy() if t.dtype != torch.bfloat16 else t.view(torch.int16).cpu().numpy().view(np.uint16)

    def sync_host():
        w.k_pool, w.v_pool = host(kvc.k_pool).copy(), host(kvc.v_pool).copy()
        if kvc.k_scale is not None:
            w.k_scale, w.v_scale = host(kvc.k_scale).copy(), host(kvc.v_scale).copy()
        w.seq_lens[:] = host(kvc.seq_lens)

    for turn in range(3):
        words = [ancestors(rng, N) for _ in range(3)]
        run = TreeRun(w, N, None, words, seed=turn)
        run.kv, run.workspace = kvc, ws
        run.scores = torch.full((3, Hkv, top), float("nan"), device=dev)
        run.run()
        torch.cuda.synchronize()
        check_tree(run, f"round {turn}")
        # a path from the root: the ancestors of one node
        path = np.zeros((3, N), dtype=np.int32)
        taken = []
        for b in range(3):
            line = [j for j in range(N) if words[b][N - 1 - b] >> j & 1]
            path[b, :len(line)] = line
            taken.append(len(line))
        scores = host(run.scores).copy()
        want = oracle.tree_commit(w, [N] * 3, path, taken, scores)
        pa.pillar_tree_commit(kvc, None, N, ints(path), ints(taken), after, run.scores)
        torch.cuda.synchronize()
        check_cache(kvc, want)
        kvc.seq_lens, after = after, kvc.seq_lens
        sync_host()
        want = oracle.evict_kv(w, host(run.scores), 0.9, host(old), [budget] * 3, 2, 8, host(weights), host(positions))
        pa.pillar_evict_kv(kvc, run.scores, 0.9, old, ints([budget] * 3), 2, 8, weights, positions, kvc.seq_lens, ws)
        torch.cuda.synchronize()
        check_cache(kvc, want)
        assert kvc.seq_lens.tolist() == want["new_lens"].tolist()
        assert np.array_equal(host(weights), want["weights"]) and np.array_equal(host(positions), want["positions"])
        old = kvc.seq_lens.clone()
        sync_host()
        # a draft step on what is left
        counts, lists, d_out = ints([0] * 3), ints(np.zeros((3, Hkv, budget))), torch.zeros(3, Hq, 128, dtype=torch.bfloat16, device=dev)
        pa.pillar_window_indices(kvc.seq_lens, ints([budget] * 3), Hkv, 0, budget, lists, counts)
        w.q_draft = gen.bf16_bits_from_f32(rng.standard_normal((3, Hq, 128), dtype=np.float32))
        q = torch.from_numpy(w.q_draft.view(np.int16)).view(torch.bfloat16).to(dev)
        pa.pillar_sparse_decode(kvc, q, lists, counts, budget, d_out, None, ws)
        torch.cuda.synchronize()
        check_out(d_out.double().cpu().numpy(), oracle.sparse_decode(w, host(lists), host(counts))[0], w.kv_dtype, f"draft {turn}")
        # the next tree's rows: N tokens that were anywhere
        room = kvc.seq_lens + N
        pages = kvc.block_table.cpu().numpy()
        for b in range(3):
            for t in range(int(kvc.seq_lens[b]), int(room[b])):
                at, frm = (pages[b, t // w.P], t % w.P), (pages[b, (t - 40) // w.P], (t - 40) % w.P)
                kvc.k_pool[at[0], :, at[1]] = kvc.k_pool[frm[0], :, frm[1]]
                kvc.v_pool[at[0], :, at[1]] = kvc.v_pool[frm[0], :, frm[1]]
        kvc.seq_lens = room.to(torch.int32)
        sync_host()
