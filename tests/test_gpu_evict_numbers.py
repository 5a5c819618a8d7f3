"""Positions of a bounded cache over many evictions, on the GPU: the number beside a row is the row's place in the text."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from tests.tree_cases import cache_of, make

pytestmark = pytest.mark.gpu

B, HKV, TOP, P = 2, 2, 120, 16


class Cache:
    """Rows of K hold the place of their token, so that a row says itself where it came from."""

    def __init__(self):
        w = make("numbers", 61, [TOP] * B, kv="f32", q="f32", Hq=HKV, Hkv=HKV, D=64, P=P)
        self.kv = cache_of(w)
        self.table, dev = w.block_table, self.kv.k_pool.device
        self.kv.seq_lens = torch.zeros(B, dtype=torch.int32, device=dev)
        self.old = torch.zeros(B, dtype=torch.int32, device=dev)
        self.weights = torch.full((B, HKV, TOP), float("nan"), device=dev)
        self.positions = torch.full((B, HKV, TOP), -5, dtype=torch.int32, device=dev)
        self.ws = torch.empty(pa.pillar_evict_workspace_bytes(self.kv), dtype=torch.uint8, device=dev)
        self.text = [0] * B
        self.rng = np.random.default_rng(7)

    def row(self, b, t):
        return self.kv.k_pool[int(self.table[b, t // P]), :, t % P]

    def append(self, counts, numbered):
        lens = self.kv.seq_lens.tolist()
        for b, n in enumerate(counts):
            for i in range(n):
                self.row(b, lens[b] + i)[:] = self.text[b] + i
                if numbered:
                    self.positions[b, :, lens[b] + i] = self.text[b] + i
                    self.weights[b, :, lens[b] + i] = 0.0
            self.text[b] += n
        self.kv.seq_lens = torch.tensor([x + n for x, n in zip(lens, counts)], dtype=torch.int32, device=self.old.device)

    def evict(self, budgets, sink, recent, numbered):
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=self.old.device)
        scores = torch.from_numpy(self.rng.random((B, HKV, TOP), dtype=np.float32)).to(self.old.device)
        now, before = ints([-1] * B), self.kv.seq_lens if numbered else self.old
        pa.pillar_evict_kv(self.kv, scores, 0.5, before, ints(budgets), sink, recent, self.weights, self.positions, now, self.ws)
        torch.cuda.synchronize()
        self.kv.seq_lens, self.old = now, now.clone()

    def check(self, sink, newest):
        for b, n in enumerate(self.kv.seq_lens.tolist()):
            for g in range(HKV):
                held = self.positions[b, g, :n].tolist()
                assert held == [int(self.row(b, t)[g, 0]) for t in range(n)]
                assert len(set(held)) == n and set(range(min(sink, n, self.text[b]))) <= set(held)
                assert not newest or n == 0 or self.text[b] - 1 in held
        assert torch.isfinite(self.weights[0, :, :int(self.kv.seq_lens[0])]).all()


STEPS = [[50, 30], [3, 70], [0, 1], [20, 5], [1, 1], [60, 2], [2, 40]]


@pytest.mark.parametrize("sink,recent,budget", [(2, 1, 3), (2, 8, 10), (0, 1, 1), (4, 16, 48), (0, 5, 40)])
def test_numbers_are_places_where_the_newest_token_stays(sink, recent, budget):
    """recent_tokens of one or more, and room for them beside the sinks."""
    c = Cache()
    for step in STEPS:
        c.append(step, False)
        c.evict([budget, budget + 5], sink, recent, False)
        c.check(sink, True)


@pytest.mark.parametrize("sink,recent,budgets", [(2, 0, [30, 12]), (2, 8, [5, 9]), (0, 0, [1, 40]), (2, 3, [2, 0])])
def test_numbers_that_the_caller_writes(sink, recent, budgets):
    """The newest token may go: new tokens come with their places, and weights of 0, and count as old ones."""
    c = Cache()
    for step in STEPS:
        c.append(step, True)
        c.evict(budgets, sink, recent, True)
        c.check(sink if min(budgets) >= sink else 0, False)
