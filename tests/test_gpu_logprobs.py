"""What rows of logits say, on the GPU, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from oracle import step_oracle as so
from tests.tree_cases import QT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Call:
    def __init__(self, x, dtype, tokens=None, top=0, scale=1.0, row_pad=0, offset=0):
        x = torch.from_numpy(np.asarray(x, dtype=np.float32)).to(QT[dtype])
        R, V = x.shape
        self.x64, self.tokens, self.top, self.scale = x.double().numpy(), tokens, top, scale
        whole = torch.full((R * (V + row_pad) + offset,), float("nan"), dtype=QT[dtype], device=DEV)
        self.logits = whole[offset:].view(R, V + row_pad)[:, :V]
        self.logits.copy_(x.to(DEV))
        nan = lambda *shape: torch.full(shape, float("nan"), device=DEV)
        self.tok = None if tokens is None else torch.tensor(tokens, dtype=torch.int32, device=DEV)
        self.lp = None if tokens is None else nan(*self.tok.shape)
        self.lse, self.entropy = nan(R), nan(R)
        self.ids = torch.full((R, top), -7, dtype=torch.int32, device=DEV) if top else None
        self.tlp = nan(R, top) if top else None
        self.workspace = torch.full((pa.pillar_logprobs_workspace_bytes(R, V, top),), 255, dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        pa.pillar_token_logprobs(self.logits, self.workspace, tokens=self.tok, logprobs=self.lp, lse=self.lse, entropy=self.entropy, top_ids=self.ids,
                                 top_logprobs=self.tlp, scale=self.scale, stream=stream)
        return self

    def check(self):
        """Alternatives are the very ones.  With n = V/64 + 80 for the additions of a lane and the joins, and u = 2^-24: the sum of exponentials is off by n u, and by
        u of every exponent; scale and log2 e are rounded into one factor, which moves a log probability by u of its distance from the mean logit (its
        own size and the entropy); lse has a rounding of its own size.  So lse is off by (n + 2 + 4 H) u + 3 u |lse| (+ u |m|), a log probability by
        (n + 4 + 4 H) u + 4 u |log p|, the entropy, a difference of log S and sum p y, by (n + 8) u (1 + H + 2 log S)."""
        want = so.logprobs(self.x64, np.float32(self.scale).astype(np.float64), None if self.tokens is None else np.asarray(self.tokens), self.top)
        R, V = self.x64.shape
        u, n = 2.0 ** -24, V / 64 + 80
        H = np.where(np.isfinite(want["entropy"]), want["entropy"], 0.0)
        finite = np.where(np.isfinite(self.x64), self.x64, -np.inf)
        m = np.abs(np.nan_to_num(finite.max(axis=1), neginf=0.0)) * self.scale
        spread = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]) + m, 0.0)
        log_s = np.log(V)

        def near(got, ref, bound, what):
            got = got.double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN"
            inf = np.isinf(ref)
            assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities"
            there = np.isfinite(ref)
            off = np.abs(got - np.where(there, ref, 0.0)) - bound
            assert not there.any() or off[there].max() <= 0, f"{what}: {off[there].max():.3g} more than its bound off"

        near(self.lse, want["lse"], (n + 2 + 4 * H) * u + 3 * u * spread, "lse")
        near(self.entropy, want["entropy"], (n + 8) * u * (1 + H + 2 * log_s), "entropy")
        each = lambda ref: (n + 4 + 4 * H)[:, None] * u + 4 * u * np.abs(np.where(np.isfinite(ref), ref, 0.0))
        if self.tok is not None:
            near(self.lp, want["logprobs"], each(want["logprobs"]), "logprobs")
        if self.top:
            assert np.array_equal(self.ids.cpu().numpy(), want["top_ids"]), "alternatives"
            near(self.tlp, want["top_logprobs"], each(want["top_logprobs"]), "top_logprobs")
        return self


def rows(R, V, seed=0, gain=3.0):
    return np.random.default_rng(seed).standard_normal((R, V)) * gain


def ids(R, V, M, seed=0):
    t = np.random.default_rng(seed + 1).integers(0, V, (R, M))
    t[0, 0] = V - 1
    return t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 255, 1000, 1024, 4097, 12345])
@pytest.mark.parametrize("top", [0, 1, 2, 20, 64])
def test_sizes(dtype, V, top):
    Call(rows(3, V, V), dtype, ids(3, V, 3), top, 1.25).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("row_pad,offset", [(0, 0), (1, 0), (3, 1), (8, 8), (0, 5), (13, 7)])
def test_strides_and_alignment(dtype, row_pad, offset):
    Call(rows(5, 3001, 2), dtype, ids(5, 3001, 1), 5, row_pad=row_pad, offset=offset).run().check()


@pytest.mark.parametrize("top", [0, 1, 8])
def test_a_long_row_and_many_rows(top):
    Call(rows(1, 100003, 3), "bf16", ids(1, 100003, 2), top).run().check()
    Call(rows(300, 2500, 4), "bf16", ids(300, 2500, 1), top).run().check()
    Call(rows(2100, 77, 5), "f32", ids(2100, 77, 1), top).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 3, 64])
@pytest.mark.parametrize("V", [500, 9000])
def test_ties_rising_and_falling(dtype, top, V):
    """Equal logits go by number; rows that rise let every logit in, rows that fall none; zeros of both signs are equal."""
    up = np.arange(V) * (8.0 / V)
    signs = np.where(np.arange(V) % 3 == 0, -0.0, 0.0)
    few = np.random.default_rng(0).integers(0, 3, V).astype(float)
    late = np.zeros(V)
    late[V - 40:] = 5.0
    Call(np.stack([np.zeros(V), up, -up, signs, few, late, up[::-1]]), dtype, ids(7, V, 2), top).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 1, 5, 64])
@pytest.mark.parametrize("V", [70, 3000])
def test_masked_logits(dtype, top, V):
    """-inf anywhere, rows of nothing else, fewer logits left than alternatives wanted."""
    x = rows(8, V, 6)
    rng = np.random.default_rng(7)
    x[0, rng.random(V) < 0.9] = -np.inf
    x[1] = -np.inf
    x[2] = -np.inf
    x[2, V // 2] = 1.5
    x[3, :V - 3] = -np.inf
    x[4, 10:] = -np.inf
    x[5, :64] = -np.inf
    x[6] = -1e30
    x[7, ::2] = -3e38
    Call(x, dtype, ids(8, V, 4), top).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 1, 5, 64])
def test_infinities_and_nan(dtype, top):
    V = 900
    x = rows(7, V, 8)
    x[0, 500] = np.inf
    x[1, [3, 800]] = np.inf
    x[2, 77] = np.nan
    x[3, 77], x[3, 78] = np.nan, np.inf
    x[4] = np.nan
    x[5] = -np.inf
    x[5, 4] = np.nan
    t = ids(7, V, 3)
    t[0, 0], t[1, 1], t[2, 2] = 500, 3, 77
    Call(x, dtype, t, top).run().check()


def test_tokens_that_are_none():
    t = np.array([[-1, 5, 1000], [999, -2147483648, 2147483647]])
    c = Call(rows(2, 1000, 9), "f32", t, 0).run().check()
    assert torch.isneginf(c.lp[0, 0]) and torch.isneginf(c.lp[0, 2]) and torch.isneginf(c.lp[1, 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_peaked_and_flat_rows(dtype):
    """One token has all but a little; all have the same; large offsets and temperatures."""
    V = 2000
    x = np.stack([np.zeros(V), np.full(V, 300.0), np.full(V, -3000.0), rows(1, V, 10)[0] + 512.0, rows(1, V, 11)[0]])
    x[4, 99] = 60.0
    for scale in (1.0, 0.01, 7.5):
        Call(x, dtype, ids(5, V, 2), 4, scale).run().check()


def test_only_what_is_asked_for():
    x = rows(4, 5000, 12)
    c = Call(x, "bf16", ids(4, 5000, 1), 6).run().check()
    alone = torch.full((4,), float("nan"), device=DEV)
    pa.pillar_token_logprobs(c.logits, c.workspace, lse=alone)
    assert torch.equal(alone, c.lse)
    pa.pillar_token_logprobs(c.logits, c.workspace, entropy=alone)
    assert torch.equal(alone, c.entropy)
    lp = torch.empty_like(c.lp)
    pa.pillar_token_logprobs(c.logits, c.workspace, tokens=c.tok, logprobs=lp)
    assert torch.equal(lp, c.lp)


def test_captured_replayed_and_two_at_once():
    calls = [Call(rows(9, 20000, s), "bf16", ids(9, 20000, 2), 8) for s in (13, 14)]
    graphs = []
    for c in calls:
        c.run().check()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outputs = lambda c: (c.lp, c.lse, c.entropy, c.ids, c.tlp)
    first = [[t.clone() for t in outputs(c)] for c in calls]
    for turn in range(4):
        for c in calls:
            for t in outputs(c):
                t.fill_(-5)
            c.workspace.fill_(turn)
        torch.cuda.synchronize()
        for g, c, s in zip(graphs, calls, streams):
            if turn % 2:
                c.run(stream=s)
            else:
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for c, f in zip(calls, first):
            assert all(torch.equal(t, was) for t, was in zip(outputs(c), f)), turn


@pytest.mark.parametrize("dtype,per", [("f32", 4), ("bf16", 8)])
@pytest.mark.parametrize("top", [1, 3, 9, 64])
def test_ties_at_the_ends_of_unaligned_rows(dtype, per, top):
    """A row's first and last logits, up to the next 16 bytes, are read apart from the others: equal ones go by number all the same."""
    V = 1500 + 3
    for offset in range(per):
        x = np.full((4, V), -1.0)
        x[0] = 0.0
        x[1, :per], x[1, 700:720], x[1, -per:] = 2.0, 2.0, 2.0
        x[2, -2:], x[2, 5] = 3.0, 3.0
        x[3, 0], x[3, 1], x[3, V - 1], x[3, 900] = 1.0, 4.0, 4.0, 4.0
        Call(x, dtype, ids(4, V, 1), top, offset=offset).run().check()


def test_entropy_is_not_negative():
    x = np.zeros((6, 3000))
    for r in range(6):
        x[r, 100 * r] = 10.0 + 7 * r
    assert (Call(x, "f32", None, 0, 3.0).run().check().entropy >= 0).all()


def test_no_rows():
    ws = torch.empty(pa.pillar_logprobs_workspace_bytes(0, 50, 2), dtype=torch.uint8, device=DEV)
    none = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device=DEV)
    pa.pillar_token_logprobs(none(0, 50), ws, tokens=none(0, 2, dtype=torch.int32), logprobs=none(0, 2), lse=none(0), top_ids=none(0, 2, dtype=torch.int32), top_logprobs=none(0, 2))
    torch.cuda.synchronize()
