"""CPU oracle for rotary positions, new tokens into the cache, their attention, and what their logits say.  TEST INFRASTRUCTURE ONLY.

Plain numpy in float64, written from the definitions in include/pillar.h.

  frequencies   angle per position of every pair, and the amplitude, for each scaling
  rotate        pairs as complex numbers times unit ones
  append_plain  rows into a cache of fp32 or bf16 values (what is stored, before its rounding)
  append_fp8    rows into a cache of 8-bit codes: scales and codes in the fp32 roundings that the definition names
  prompt_attn   causal softmax attention of packed new tokens; beside the results what rounding errors are proportional to
  logprobs      log-sum-exp, log probabilities, entropy, the tokens of largest logit
"""
from __future__ import annotations

import math

import numpy as np

from .pillar_oracle import e4m3_table, gather_request

__all__ = ["frequencies", "rotate", "token_of_row", "append_plain", "append_fp8", "encode_e4m3", "prompt_attn", "logprobs"]

_TABLE = e4m3_table()
_GRID = _TABLE[:127]                                     # values of the codes 0..126, ascending; 127 is NaN


def frequencies(r, base, scaling="none", factor=1.0, original_len=0, fast=0.0, slow=0.0):
    f, amplitude = [], 1.0
    if scaling == "base":
        base = base * factor ** (r / max(r - 2, 1))
    for i in range(r // 2):
        own = base ** (-2.0 * i / r)
        if scaling == "linear":
            own /= factor
        elif scaling == "ramp":
            at = lambda turns: r * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))
            low, high = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), r - 1)
            share = min(max((i - low) / max(high - low, 0.001), 0.0), 1.0)
            own = own * (1 - share) + own / factor * share
            amplitude = 0.1 * math.log(factor) + 1.0
        elif scaling == "bands":
            share = min(max((original_len * own / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0)
            own = own * share + own / factor * (1 - share)
        f.append(own)
    return np.array(f), amplitude


def rotate(x, positions, f, amplitude=1.0, interleaved=False):
    """x: float64 [T, H, D]; positions: [T]."""
    y = np.array(x, dtype=np.float64)
    m = len(f)
    one, two = (np.arange(m) * 2, np.arange(m) * 2 + 1) if interleaved else (np.arange(m), np.arange(m) + m)
    unit = amplitude * np.exp(1j * np.asarray(positions, dtype=np.float64)[:, None, None] * f)
    z = (y[..., one] + 1j * y[..., two]) * unit
    y[..., one], y[..., two] = z.real, z.imag
    return y


def token_of_row(seq_lens, starts):
    """(request, token) of every packed row."""
    return [(b, int(seq_lens[b]) - (starts[b + 1] - starts[b]) + i) for b in range(len(seq_lens)) for i in range(starts[b + 1] - starts[b])]


def append_plain(w, pool, rows, starts):
    """pool: float64 [pages, Hkv, P, D], changed; rows: float64 [T, Hkv, D]."""
    for r, (b, t) in enumerate(token_of_row(w.seq_lens, starts)):
        if t >= 0:
            pool[w.block_table[b, t // w.P], :, t % w.P] = rows[r]


def encode_e4m3(x):
    """Nearest code of float64 values within +-448, ties to the even code; NaN to 127."""
    x = np.asarray(x, dtype=np.float64)
    m = np.abs(x)
    hi = np.clip(np.searchsorted(_GRID, np.nan_to_num(m)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    near = np.where(_GRID[hi] - m < m - _GRID[lo], hi, lo)
    tie = _GRID[hi] - m == m - _GRID[lo]
    near = np.where(tie, np.where(hi % 2 == 0, hi, lo), near)
    near = np.where(m >= _GRID[126], 126, near)
    return np.where(np.isnan(x), 127, near + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def append_fp8(w, pool, scale, rows, starts):
    """pool: uint8 codes [pages, Hkv, P, D], scale: fp32 [pages, Hkv], both changed; rows: fp32 [T, Hkv, D], as the page is to hold them."""
    f32 = np.float32
    by_page = {}
    for r, (b, t) in enumerate(token_of_row(w.seq_lens, starts)):
        if t >= 0:
            by_page.setdefault((b, t // w.P), []).append((t % w.P, r))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for (b, p), new in by_page.items():
            page, older = w.block_table[b, p], new[0][0]
            for g in range(rows.shape[1]):
                x = np.stack([rows[r, g] for _, r in new]).astype(f32)
                most = np.abs(x[np.isfinite(x)]).max(initial=f32(0))
                fresh = f32(0) if most < f32(2.0 ** -90) else f32(most / f32(448))
                had = scale[page, g]
                now = max(had, fresh) if older > 0 else fresh
                if older > 0 and now != had:
                    ratio = f32(had / now)
                    pool[page, g, :older] = encode_e4m3((_TABLE[pool[page, g, :older]].astype(f32) * ratio).astype(f32))
                inv = f32(0) if now < f32(f32(2.0 ** -90) / f32(448)) else f32(f32(1) / now)
                y = (x * inv).astype(f32)
                y = np.where(np.abs(y) > 448, np.copysign(f32(448), y), y)
                for i, (slot, _) in enumerate(new):
                    pool[page, g, slot] = encode_e4m3(y[i])
                scale[page, g] = now


def prompt_attn(w, q, starts):
    """q: float64 [T, Hq, D].  Rows past starts[B] hold NaN in the results.  Beside out and lse: weight = sum p |v|, reach = the largest sum |q k| of a logit."""
    T, Hq, D = q.shape
    G = Hq // w.Hkv
    out, weight, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    reach = 0.0
    for b in range(w.B):
        L, n = int(w.seq_lens[b]), starts[b + 1] - starts[b]
        k, v = gather_request(w, b) if L > 0 else (np.zeros((0, w.Hkv, D)), np.zeros((0, w.Hkv, D)))
        for i in range(n):
            r, sees = starts[b] + i, max(0, L - n + i + 1)
            for h in range(Hq):
                if sees == 0:
                    out[r, h], weight[r, h], lse[r, h] = 0.0, 0.0, -np.inf
                    continue
                kk, vv = k[:sees, h // G], v[:sees, h // G]
                s = (kk @ q[r, h]) * w.sm_scale
                reach = max(reach, float((np.abs(kk) @ np.abs(q[r, h])).max()) * w.sm_scale)
                m = s.max()
                p = np.exp(s - m)
                lse[r, h] = m + np.log(p.sum())
                p /= p.sum()
                out[r, h] = p @ vv
                weight[r, h] = p @ np.abs(vv)
    return {"out": out, "lse": lse, "weight": weight, "reach": reach}


def logprobs(x, scale, tokens=None, top=0):
    """x: float64 [R, V]; tokens: [R, M]."""
    R, V = x.shape
    M = 0 if tokens is None else tokens.shape[1]
    res = {"lse": np.zeros(R), "entropy": np.zeros(R), "logprobs": np.zeros((R, M)), "top_ids": np.full((R, top), -1), "top_logprobs": np.full((R, top), -np.inf)}
    for r in range(R):
        z = x[r] * scale
        if np.isnan(z).any():
            lse = entropy = np.nan
            lp = np.full(V, np.nan)
        elif (z == np.inf).any():
            lse, entropy = np.inf, np.nan
            lp = np.where(z == np.inf, np.nan, -np.inf)
        elif (z == -np.inf).all():
            lse, entropy, lp = -np.inf, 0.0, z
        else:
            log_sum = np.log(np.exp(z - z.max()).sum())
            lse = z.max() + log_sum
            lp = (z - z.max()) - log_sum                 # (not z - lse: logits of -1e30 have no room for log V beside them)
            p = np.exp(lp)
            entropy = -(p[p > 0] * lp[p > 0]).sum()
        res["lse"][r], res["entropy"][r] = lse, entropy
        for j in range(M):
            id = int(tokens[r, j])
            res["logprobs"][r, j] = lp[id] if 0 <= id < V else -np.inf
        order = sorted(range(V), key=lambda i: (np.isnan(x[r, i]), -x[r, i] if not np.isnan(x[r, i]) else 0.0, i))[:top]
        res["top_ids"][r, :len(order)], res["top_logprobs"][r, :len(order)] = order, lp[order]
    return res
