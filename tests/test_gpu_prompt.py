"""Attention of new tokens on the GPU, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from oracle import step_oracle as so
from tests.tree_cases import QT, TreeRun, cache_of, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GENERIC = pa.PILLAR_FLAG_GENERIC_KERNELS


class PromptRun:
    """Device tensors of one call; outputs start as NaN, with rows behind the last request's."""

    def __init__(self, w, new, seed=0, flags=0, pad=2, gain=1.0):
        rng = np.random.default_rng(seed)
        self.w, self.new = w, new
        self.starts = [sum(new[:b]) for b in range(len(new) + 1)]
        T = self.starts[-1] + pad
        q = torch.from_numpy(gain * rng.standard_normal((T, w.Hq, w.D)).astype(np.float32)).to(QT[w.q_dtype])
        self.q64, self.q = q.double().numpy(), q.to(DEV)
        self.kv = cache_of(w, flags)
        self.most = max(max(new), 1)
        self.out = torch.full((T, w.Hq, w.D), float("nan"), dtype=QT[w.q_dtype], device=DEV)
        self.lse = torch.full((T, w.Hq), float("nan"), device=DEV)
        self.starts_dev = torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        self.workspace = torch.full((pa.pillar_prompt_workspace_bytes(self.kv, T, self.most),), 255, dtype=torch.uint8, device=DEV)

    def run(self, with_lse=True, stream=None):
        pa.pillar_prompt_attn(self.kv, self.q, self.most, self.out, self.lse if with_lse else None, self.workspace, starts=self.starts_dev, stream=stream)


def check_prompt(run, what=""):
    """As tests/tree_cases.py's check_tree, whose bounds these are: a logit is off by D 2^-24 of sum |q k|, a probability by twice that and what sums over
    L tokens add, matrix cores that take bf16 round a probability by 2^-8 of itself, the output's own rounding is 2^-8 (bf16) or 2^-24 of it."""
    w = run.w
    want = so.prompt_attn(w, run.q64, run.starts)
    out, lse = run.out.double().cpu().numpy(), run.lse.double().cpu().numpy()
    L, u = int(max(w.seq_lens.max(), 1)), 2.0 ** -24
    logit = w.D * u * want["reach"]
    prob = 2 * logit + (L + 32) * u
    half = 2.0 ** -8 if w.q_dtype == "bf16" else u
    taken = 2.0 ** -8 if w.q_dtype == "bf16" and w.kv_dtype != "f32" else 0.0
    assert np.array_equal(np.isnan(out), np.isnan(want["out"])), f"{what}: not the rows that are there were written, or NaN among them"
    there = ~np.isnan(want["out"])
    fine = there & np.isfinite(want["out"])
    assert np.array_equal(out[there & ~fine], want["out"][there & ~fine]), f"{what}: infinities"
    with np.errstate(invalid="ignore"):
        bound = (taken + prob) * want["weight"] + half * np.abs(want["out"]) + 1e-30
        worst = (np.abs(out - want["out"]) / bound)[fine].max() if fine.any() else 0.0
    assert worst <= 1.0, f"{what}: out is {worst:.3g} times its bound off"
    there = ~np.isnan(want["lse"])
    assert np.array_equal(np.isnan(lse), ~there), f"{what}: lse"
    assert np.array_equal(np.isneginf(lse), np.isneginf(want["lse"])), f"{what}: lse of rows that see nothing"
    there &= np.isfinite(want["lse"])
    off = np.abs(lse[there] - want["lse"][there]) - (logit + (L + 8) * u + 8 * u * np.abs(want["lse"][there]))
    assert not there.any() or off.max() <= 0, f"{what}: lse off by {off.max():.3g} more than its bound"


TYPES = [("bf16", "bf16"), ("bf16", "fp8_e4m3"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "fp8_e4m3")]
SHAPES = [
    dict(lens=[1], new=[1]), dict(lens=[64], new=[64]), dict(lens=[65, 2], new=[65, 1]), dict(lens=[200, 131, 17], new=[1, 1, 1]),
    dict(lens=[300, 40, 129], new=[70, 33, 129]), dict(lens=[100, 7, 60], new=[0, 7, 2]), dict(lens=[5, 90], new=[40, 3]),        # (more new rows than tokens)
    dict(lens=[0, 30, 0], new=[3, 5, 0]),                                                                                          # (no token at all)
]


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 1), (128, 2, 2)])
def test_prompt(q, kv, shape, D, Hq, Hkv):
    r = PromptRun(make("prompt", 21, shape["lens"], Hq=Hq, Hkv=Hkv, D=D, q=q, kv=kv), shape["new"])
    r.run()
    check_prompt(r)


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 16])
@pytest.mark.parametrize("new", [[1, 1], [3, 9], [40, 5], [150, 70]])
def test_groups(G, new, flags):
    """Every shape of a workgroup: up to 32, 64, 128 and 256 rows of a tile, groups that fill them and groups that do not."""
    r = PromptRun(make("groups", 22, [n + m for n, m in zip(new, (90, 3))], Hq=G, Hkv=1, D=64), new, flags=flags)
    r.run()
    check_prompt(r)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("P", [1, 2, 16, 64, 256])
def test_pages(kv, P):
    r = PromptRun(make("pages", 23, [333, 65], Hq=4, Hkv=2, D=128, P=P, kv=kv), [200, 65])
    r.run()
    check_prompt(r)


def test_large_enough_for_tiles_of_256_rows():
    """Many units, so that bf16 takes eight wavefronts to a tile: whole prompts, a chunk, single tokens."""
    for kv in ("bf16", "fp8_e4m3"):
        new = [600, 1, 333, 256, 1, 64]
        r = PromptRun(make("tiles", 24, [600, 1500, 900, 256, 70, 1100], Hq=16, Hkv=4, D=128, kv=kv), new)
        r.most = 600
        r.run()
        check_prompt(r, kv)


def test_one_long_prompt_is_split_and_joined():
    r = PromptRun(make("long", 25, [2500], Hq=2, Hkv=1, D=64), [40])
    r.run()
    check_prompt(r)
    r = PromptRun(make("long", 26, [4000, 3900], Hq=4, Hkv=1, D=128), [1, 1])
    r.run()
    check_prompt(r)


def test_many_requests():
    rng = np.random.default_rng(27)
    new = [int(n) for n in rng.integers(0, 6, 150)]
    r = PromptRun(make("many", 27, [int(m) + n for n, m in zip(new, rng.integers(0, 60, 150))], Hq=2, Hkv=1, D=64), new)
    r.run()
    check_prompt(r)


def test_chains_give_what_the_tree_gives():
    """The same tokens as a chain of a tree: two kernels, one definition."""
    w = make("chain", 28, [500, 260, 33], Hq=8, Hkv=2, D=128)
    N = 20
    tree = TreeRun(w, N, None, [[2 ** (i + 1) - 1 for i in range(N)]] * 3, seed=3)
    tree.run(with_scores=False)
    r = PromptRun(w, [N] * 3, pad=0)
    r.q.copy_(tree.q.reshape(r.q.shape))
    r.run()
    # each is within its own bound of the definition; both round P (2^-8) and the output (2^-8): at most twice the sum of both of what is summed
    gap = (r.out.double() - tree.out.double().reshape(r.out.shape)).abs()
    assert gap.max() <= 4 * 2.0 ** -8 * tree.out.double().abs().max() + 1e-6
    assert (r.lse - tree.lse.reshape(r.lse.shape)).abs().max() <= 1e-4


def test_what_is_not_seen_has_no_influence():
    """Infinities and NaN in K and V of later tokens: earlier rows keep their bits, those that see them get what the definition says."""
    for q, kv in (("bf16", "bf16"), ("f32", "f32"), ("bf16", "fp8_e4m3"), ("f32", "bf16")):
        w = make("masked", 29, [150, 90], Hq=4, Hkv=2, D=64, q=q, kv=kv)
        clean = PromptRun(w, [100, 90])
        clean.run()
        dirty = PromptRun(w, [100, 90])
        put = {"bf16": [float("inf"), float("nan")], "f32": [float("inf"), float("nan")], "fp8_e4m3": [127, 255]}[kv]
        for b, t in ((0, 97), (0, 120), (1, 60)):
            page, slot = int(w.block_table[b, t // w.P]), t % w.P
            dirty.kv.v_pool[page, :, slot, 5] = put[0]
            dirty.kv.k_pool[page, :, slot, 3] = put[1]
        dirty.run()
        for b, t in ((0, 97), (1, 60)):                    # the first dirty token of each request
            lo, own = clean.starts[b], clean.starts[b] + t - (int(w.seq_lens[b]) - clean.new[b])
            assert torch.equal(clean.out[lo:own], dirty.out[lo:own]) and torch.equal(clean.lse[lo:own], dirty.lse[lo:own])
            assert torch.isnan(dirty.out[own:clean.starts[b + 1]]).all()
        # V alone: one dim of the rows that see it is infinite or no number, the others as they were
        only_v = PromptRun(w, [100, 90])
        page, slot = int(w.block_table[0, 97 // w.P]), 97 % w.P
        only_v.kv.v_pool[page, :, slot, 5] = put[0]
        only_v.run()
        own = clean.starts[0] + 97 - 50
        assert torch.equal(clean.out[:own], only_v.out[:own]) and torch.equal(clean.lse[:190], only_v.lse[:190])
        assert not torch.isfinite(only_v.out[own:100, :, 5].float()).any()
        rest = [d for d in range(64) if d != 5]
        assert torch.equal(clean.out[:190][:, :, rest], only_v.out[:190][:, :, rest])


def test_strides_alignment_and_the_generic_kernels():
    w = make("strides", 30, [140, 77], Hq=4, Hkv=2, D=64)
    plain = PromptRun(w, [90, 77])
    plain.run()
    strided = PromptRun(w, [90, 77])
    for name in ("k_pool", "v_pool"):
        p = getattr(strided.kv, name)
        wide = torch.zeros(p.shape[0], p.shape[2], p.shape[1], 72, dtype=p.dtype, device=DEV)
        wide[..., :64].transpose(1, 2).copy_(p)
        setattr(strided.kv, name, wide[..., :64].transpose(1, 2))
    strided.run()
    assert torch.equal(plain.out[:167], strided.out[:167]) and torch.equal(plain.lse[:167], strided.lse[:167])
    odd = PromptRun(w, [90, 77])                           # rows at odd distances: one element at a time
    for name in ("k_pool", "v_pool"):
        p = getattr(odd.kv, name)
        wide = torch.zeros(p.shape[0], p.shape[1], p.shape[2], 67, dtype=p.dtype, device=DEV)
        wide[..., 1:65].copy_(p)
        setattr(odd.kv, name, wide[..., 1:65])
    odd.run()
    check_prompt(odd)
    generic = PromptRun(w, [90, 77], flags=GENERIC)
    generic.run()
    check_prompt(generic)


def test_without_starts_and_without_lse():
    w = make("even", 31, [140, 77], Hq=4, Hkv=2, D=64)
    a, b = PromptRun(w, [30, 30], pad=0), PromptRun(w, [30, 30], pad=0)
    a.run()
    pa.pillar_prompt_attn(b.kv, b.q, 30, b.out, None, b.workspace)
    assert torch.equal(a.out, b.out)
    check_prompt(a)


def test_large_logits_and_large_scales():
    """Rows dominated by one token, and scales of pages far apart."""
    r = PromptRun(make("sharp", 32, [300, 128], Hq=4, Hkv=2, D=64, kv="fp8_e4m3"), [200, 128], gain=20.0)
    r.run()
    check_prompt(r)
    w = make("scales", 33, [300, 128], Hq=4, Hkv=2, D=64, kv="fp8_e4m3")
    with np.errstate(invalid="ignore"):
        w.v_scale *= (2.0 ** np.random.default_rng(0).integers(-20, 12, w.v_scale.shape)).astype(np.float32)
    r = PromptRun(w, [200, 128])
    r.run()
    check_prompt(r)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_captured_replayed_and_two_at_once(kv):
    ws = [make("graph", s, [700, 300], Hq=8, Hkv=2, D=128, kv=kv) for s in (34, 35)]
    runs = [PromptRun(w, [300, 20], seed=i) for i, w in enumerate(ws)]
    for r in runs:
        r.run()
    torch.cuda.synchronize()
    first = [(r.out.clone(), r.lse.clone()) for r in runs]
    for r in runs:
        check_prompt(r)
    graphs = []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.run()
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for r in runs:
            r.out.fill_(float("nan")), r.lse.fill_(float("nan")), r.workspace.fill_(turn)
        torch.cuda.synchronize()
        for g, r, s in zip(graphs, runs, streams):
            if turn % 2:
                r.run(stream=s)
            else:
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for r, (out, lse) in zip(runs, first):
            assert torch.equal(r.out[:320], out[:320]) and torch.equal(r.lse[:320], lse[:320]) and torch.isnan(r.out[320:]).all(), turn


def test_a_workspace_asked_for_more_does_for_less():
    w = make("less", 36, [700, 300], Hq=8, Hkv=2, D=128)
    r = PromptRun(w, [300, 20])
    small = PromptRun(w, [1, 1])
    small.workspace = r.workspace
    small.run()
    check_prompt(small)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (32, 2), (10, 2)])
def test_few_rows_among_prompts(kv, Hq, Hkv):
    """Requests on both sides of what counts as few rows, cut into ranges at any place."""
    G = Hq // Hkv
    new = [1, 64 // G, 64 // G + 1, 300, 2, 0, 150, 1]
    r = PromptRun(make("few", 37, [1900, 700, 64 // G + 1, 300, 5, 40, 950, 1], Hq=Hq, Hkv=Hkv, D=128, kv=kv), new)
    r.run()
    check_prompt(r)


def test_no_rows_and_no_tokens():
    w = make("none", 38, [5, 9], Hq=4, Hkv=2, D=64)
    r = PromptRun(w, [0, 0])
    r.run()
    assert torch.isnan(r.out).all() and torch.isnan(r.lse).all()
    pa.pillar_prompt_attn(r.kv, r.q[:0], 1, r.out[:0], None, r.workspace, starts=r.starts_dev)
    empty = PromptRun(make("empty", 39, [0, 0, 0], Hq=4, Hkv=2, D=64), [3, 0, 40])
    empty.run()
    check_prompt(empty)


def test_bounds_that_are_far_above_the_lengths():
    """max_seq_len and max_new choose kernels, and change nothing else."""
    w = make("bounds", 40, [300, 40, 129], Hq=8, Hkv=2, D=64, extra_table_cols=600)
    for most in (70, 5000):
        r = PromptRun(w, [70, 33, 9])
        r.kv.max_seq_len = 9000
        r.most = most
        r.workspace = torch.empty(pa.pillar_prompt_workspace_bytes(r.kv, r.q.shape[0], most), dtype=torch.uint8, device=DEV)
        r.run()
        check_prompt(r, str(most))


def test_queries_and_results_at_any_address():
    """Rows that are not at multiples of 16 bytes: fp32 arithmetic, one element at a time."""
    r = PromptRun(make("address", 41, [90, 33], Hq=4, Hkv=2, D=64), [50, 33])
    for name in ("q", "out"):
        t = getattr(r, name)
        at = torch.full((t.numel() + 3,), float("nan"), dtype=t.dtype, device=DEV)[3:].view(t.shape)
        at.copy_(t)
        setattr(r, name, at)
    r.run()
    check_prompt(r)


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_replayed_with_other_lengths(kv):
    """Lengths and starts are on the device: a captured call works out its share of the work anew."""
    w = make("lengths", 42, [900, 500, 40, 300], Hq=16, Hkv=4, D=128, kv=kv)
    r = PromptRun(w, [300, 1, 40, 64])
    r.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.run()
    for lens, new in (([900, 500, 40, 300], [300, 1, 40, 64]), ([17, 400, 0, 299], [2, 280, 3, 100]), ([880, 1, 33, 64], [0, 1, 33, 64])):
        w.seq_lens[:] = lens
        r.starts = [sum(new[:b]) for b in range(5)]
        r.kv.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        r.starts_dev.copy_(torch.tensor(r.starts, dtype=torch.int32))
        r.out.fill_(float("nan")), r.lse.fill_(float("nan")), r.workspace.fill_(77)
        g.replay()
        torch.cuda.synchronize()
        check_prompt(r, str(lens))
