"""Shared helpers of the tests of trees and of the bounded cache: random trees, uploads, tolerances."""
from __future__ import annotations

import numpy as np
import torch

import gen
import oracle
import paper_2512_01278_amd as pa

QT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ancestors(rng, n, reach=8):
    """Words of a random tree: node i and its ancestors."""
    words = []
    for i in range(n):
        p = int(rng.integers(max(-1, i - reach), i)) if i else -1
        words.append((words[p] if p >= 0 else 0) | 1 << i)
    return words


def as_int64(words):
    """Python integers of 64 bits -> the int64 tensor of the same bits."""
    return torch.from_numpy(np.array([[x & (2 ** 64 - 1) for x in row] for row in words], dtype=np.uint64).view(np.int64))


def cache_of(w, flags=0, device="cuda:0"):
    kv = pa.upload_workload(w, device).kv
    kv.flags = flags
    kv.max_seq_len = max(1, kv.max_seq_len)
    return kv


def make(name, seed, lens, *, Hq=8, Hkv=2, D=128, P=16, q="bf16", kv="bf16", **more):
    lens = np.asarray(lens)
    w = gen.make_custom(name=name, seed=seed, B=len(lens), Hq=Hq, Hkv=Hkv, D=D, P=P, spec_k=0, q_dtype=q, kv_dtype=kv, seq_lens=np.maximum(lens, 1),
                        budgets=[1] * len(lens), sink_tokens=2, **more)
    w.seq_lens[:] = lens
    return w


def queries(rng, w, N):
    """Host queries as stored values, and what they stand for in float64."""
    x = rng.standard_normal((w.B, N, w.Hq, w.D), dtype=np.float32)
    if w.q_dtype == "f32":
        return torch.from_numpy(x), x.astype(np.float64)
    bits = gen.bf16_bits_from_f32(x)
    return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16), gen.f32_from_bf16_bits(bits).astype(np.float64)


class TreeRun:
    """Device tensors of one verification of trees; outputs start as NaN."""

    def __init__(self, w, N, sizes, words, seed=0, flags=0, queries_of=None):
        rng = np.random.default_rng(seed)
        q, self.q64 = queries(rng, w, N) if queries_of is None else queries_of
        self.w, self.N, self.words = w, N, words
        self.sizes = np.full(w.B, N) if sizes is None else np.asarray(sizes)
        self.kv = cache_of(w, flags)
        dev = self.kv.k_pool.device
        self.q, self.visible = q.to(dev), as_int64(words).to(dev)
        self.sizes_dev = None if sizes is None else torch.tensor(self.sizes, dtype=torch.int32, device=dev)
        nan = lambda *shape, dtype=torch.float32: torch.full(shape, float("nan"), dtype=dtype, device=dev)
        self.out = nan(w.B, N, w.Hq, w.D, dtype=QT[w.q_dtype])
        self.lse = nan(w.B, N, w.Hq)
        self.scores = nan(w.B, w.Hkv, self.kv.max_seq_len + 3)
        self.workspace = torch.empty(pa.pillar_tree_workspace_bytes(self.kv, N), dtype=torch.uint8, device=dev)

    def run(self, with_lse=True, with_scores=True, stream=None):
        pa.pillar_verify_tree(self.kv, self.q, self.sizes_dev, self.visible, self.out, self.lse if with_lse else None,
                              self.scores if with_scores else None, self.workspace, stream=stream)


def check_tree(run, what, with_scores=True):
    """Against the oracle, element by element.

    Errors are bounded from the arithmetic.  A logit is a sum of D products of at most `reach` in all: each of its roundings is off by 2^-24 of that at
    most, so the logit by D 2^-24 reach, and a probability, which has its own logit and the log-sum-exp in its exponent, by twice that, plus
    what the sums over L tokens and the exponential add (2^-24 each).  Matrix cores that take bf16 round a probability by 2^-8 of itself, twice
    nothing: the output by 2^-8 of sum p |v|.  The output's own rounding is 2^-8 (bf16) or 2^-24 of it."""
    w = run.w
    want = oracle.verify_tree(w, run.q64, run.sizes, run.words)
    out, lse, scores = (t.double().cpu().numpy() for t in (run.out, run.lse, run.scores))
    L = int(w.seq_lens.max())
    u = 2.0 ** -24
    logit = w.D * u * want["reach"]
    prob = 2 * logit + (L + 32) * u
    half = 2.0 ** -8 if w.q_dtype == "bf16" else u
    taken = 2.0 ** -8 if w.q_dtype == "bf16" and w.kv_dtype != "f32" else 0.0
    assert np.array_equal(np.isnan(out), np.isnan(want["out"])), f"{what}: not the rows that are there were written, or NaN among them"
    there = ~np.isnan(want["out"])
    fine = there & np.isfinite(want["out"])
    assert np.array_equal(out[there & ~fine], want["out"][there & ~fine]), f"{what}: infinities"
    bound = (taken + prob) * want["weight"] + half * np.abs(want["out"]) + 1e-30
    with np.errstate(invalid="ignore"):
        worst = (np.abs(out - want["out"]) / bound)[fine].max() if fine.any() else 0.0
    assert worst <= 1.0, f"{what}: out is {worst:.3g} times its bound off"
    there = ~np.isnan(want["lse"])
    assert np.array_equal(np.isnan(lse), ~there), f"{what}: lse"
    assert np.array_equal(np.isneginf(lse), np.isneginf(want["lse"])), f"{what}: lse of rows that see nothing"
    there &= np.isfinite(want["lse"])
    off = np.abs(lse[there] - want["lse"][there]) - (logit + (L + 8) * u + 8 * u * np.abs(want["lse"][there]))
    assert not there.any() or off.max() <= 0, f"{what}: lse off by {off.max():.3g} more than its bound"
    if with_scores:
        got = scores[:, :, :want["scores"].shape[2]]
        there = ~np.isnan(want["scores"])
        assert np.array_equal(np.isnan(got), ~there) and np.isnan(scores[:, :, want["scores"].shape[2]:]).all(), f"{what}: scores written where there is no token"
        biggest = np.abs(want["lse"][np.isfinite(want["lse"])]).max(initial=0.0)
        rel = prob + (run.N * w.G + 16 * (1 + biggest)) * u
        off = np.abs(got[there] - want["scores"][there]) - rel * want["scores"][there] - 1e-36
        assert not there.any() or off.max() <= 0, f"{what}: scores off by {off.max():.3g} more than their bound"
    return worst
