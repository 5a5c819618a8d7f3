"""CPU oracle for trees of drafted tokens and for the bounded cache.  TEST INFRASTRUCTURE ONLY.

Plain numpy in float64, written from the definitions in include/pillar.h, with loops over requests and heads.

  verify_tree  softmax attention of every node over the tokens before the tree and the nodes that its word names; the statistic is
               the mean of the probabilities over the nodes and the heads of a group.  Beside the results it returns what the
               rounding errors of fp32 and bf16 arithmetic are proportional to: sum p |v| and the largest sum |q k| of a logit.
  tree_commit  rows of the accepted path become the end of the context.
  evict_kv     weights are accumulated, the budget is kept, what stays beyond it moves into the freed slots.

The moves are integer-exact, and so are the weights: the formula names two fp32 roundings.  An fp8 row that changes pages is
encoded anew against the largest scale among the rows that its new page then has.
"""
from __future__ import annotations

import numpy as np

from .pillar_oracle import e4m3_table, gather_request

__all__ = ["verify_tree", "tree_commit", "evict_kv"]

_TABLE = e4m3_table()
_FINITE = np.flatnonzero(~np.isnan(_TABLE[:128]))        # codes of the values >= 0, ascending


def verify_tree(w, q, sizes, words):
    """q: float64 [B, N, Hq, D]; sizes: [B]; words: [B][N] Python integers.  Slots past a request's size hold NaN in the results, scores past
    its length too."""
    B, N, Hq, D = q.shape
    Hkv = w.Hkv
    G = Hq // Hkv
    top = max(1, int(w.seq_lens.max()))
    out, weight = np.full((B, N, Hq, D), np.nan), np.full((B, N, Hq, D), np.nan)
    lse, scores = np.full((B, N, Hq), np.nan), np.full((B, Hkv, top), np.nan)
    reach = 0.0
    for b in range(B):
        L, n = int(w.seq_lens[b]), int(sizes[b])
        if n == 0:
            continue
        k, v = gather_request(w, b)
        first = L - n
        sees = np.zeros((n, L), dtype=bool)
        for i in range(n):
            for t in range(L):
                sees[i, t] = t < first or bool(words[b][i] >> (t - first) & 1)
        for g in range(Hkv):
            rows = q[b, :n, g * G:(g + 1) * G].reshape(n * G, D)
            mask = np.repeat(sees, G, axis=0)
            total = np.zeros(L)
            for r in range(n * G):
                at = (b, r // G, g * G + r % G)
                seen = np.flatnonzero(mask[r])
                if len(seen) == 0:
                    out[at], weight[at], lse[at] = 0.0, 0.0, -np.inf
                    continue
                s = (k[seen, g] @ rows[r]) * w.sm_scale
                reach = max(reach, float((np.abs(k[seen, g]) @ np.abs(rows[r])).max()) * w.sm_scale)
                m = s.max()
                p = np.exp(s - m)
                lse[at] = m + np.log(p.sum())
                p = p / p.sum()
                with np.errstate(invalid="ignore", over="ignore"):
                    out[at] = p @ v[seen, g]
                    weight[at] = p @ np.abs(v[seen, g])
                total[seen] += p
            scores[b, g, :L] = total / (n * G)
    return {"out": out, "lse": lse, "scores": scores, "weight": weight, "reach": reach}


def _encode(x):
    """float32 -> e4m3 code: the nearest value, ties to the even code."""
    code = np.searchsorted((_TABLE[_FINITE][1:] + _TABLE[_FINITE][:-1]) / 2, np.abs(x).astype(np.float64), side="left")
    half = (_TABLE[_FINITE][1:] + _TABLE[_FINITE][:-1]) / 2
    tie = (code < len(half)) & (np.abs(x).astype(np.float64) == half[np.minimum(code, len(half) - 1)]) & (code % 2 == 1)
    code = np.where(np.isnan(x), 0x7F, code + tie)
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def _recode(codes, had, now):
    if had == now:
        return codes
    return _encode(_TABLE[codes].astype(np.float32) * np.float32(np.float32(had) / np.float32(now)))


def _move(w, pools, b, g, src, dst, live):
    """Rows src of (request, head) become rows dst, all read before any is written; `live` tokens count afterwards."""
    P = w.P
    page = lambda t: int(w.block_table[b, t // P])
    for name in ("k", "v"):
        pool, scale = pools[name + "_pool"], pools.get(name + "_scale")
        rows = [pool[page(t), g, t % P].copy() for t in src]
        if scale is None:
            for row, t in zip(rows, dst):
                pool[page(t), g, t % P] = row
            continue
        had = [scale[page(t), g] for t in src]
        to_page = {}
        for row, s, t in zip(rows, had, dst):
            to_page.setdefault(t // P, []).append((row, s, t))
        new = {}
        for p, arrivals in to_page.items():
            gone = {t for _, _, t in arrivals}
            stay = [t for t in range(p * P, min((p + 1) * P, live)) if t not in gone]
            old = scale[page(p * P), g]
            new[p] = max([s for _, s, _ in arrivals] + ([old] if stay else []))
            for t in stay:
                pool[page(t), g, t % P] = _recode(pool[page(t), g, t % P], old, new[p])
            for row, s, t in arrivals:
                pool[page(t), g, t % P] = _recode(row, s, new[p])
        for p, s in new.items():
            scale[page(p * P), g] = s


def _pools(w):
    r = {"k_pool": w.k_pool.copy(), "v_pool": w.v_pool.copy()}
    if w.k_scale is not None:
        r.update(k_scale=w.k_scale.copy(), v_scale=w.v_scale.copy())
    return r


def tree_commit(w, sizes, path, path_lens, scores=None):
    """path: [B][M].  Returns the pools (and scores), and the new lengths."""
    r = _pools(w)
    r["new_lens"] = np.zeros(w.B, dtype=np.int32)
    if scores is not None:
        r["scores"] = scores.copy()
    for b in range(w.B):
        first = int(w.seq_lens[b]) - int(sizes[b])
        nodes = []
        for i in range(max(0, min(int(path_lens[b]), path.shape[1]))):
            if first < 0 or not 0 <= path[b, i] < sizes[b]:
                break
            nodes.append(int(path[b, i]))
        r["new_lens"][b] = max(first, 0) + len(nodes)
        src, dst = [first + j for j in nodes], [first + i for i in range(len(nodes))]
        for g in range(w.Hkv):
            _move(w, r, b, g, src, dst, first + len(nodes))
            if scores is not None:
                r["scores"][b, g, dst] = scores[b, g, src]
    return r


def evict_kv(w, scores, decay, old_lens, budgets, sink, recent, weights, positions):
    r = _pools(w)
    r["weights"], r["positions"] = weights.copy(), positions.copy()
    r["new_lens"] = np.zeros(w.B, dtype=np.int32)
    for b in range(w.B):
        L = int(w.seq_lens[b])
        o = min(max(int(old_lens[b]), 0), L)
        keep = min(max(int(budgets[b]), 0), L)
        r["new_lens"][b] = keep
        for g in range(w.Hkv):
            now = np.zeros(L, dtype=np.float32)
            if scores is not None:
                now[:] = scores[b, g, :L]
                now[:o] = (weights[b, g, :o] * np.float32(decay)).astype(np.float32) + scores[b, g, :o]
            else:
                now[:o] = weights[b, g, :o]
            last = int(positions[b, g, :o].max()) if o else -1
            came = np.concatenate([positions[b, g, :o].astype(np.int64), last + 1 + np.arange(L - o)])
            newest = last + L - o
            order = sorted(range(L), key=lambda t: (not (came[t] < sink or came[t] > newest - recent),
                                                    0.0 if came[t] < sink or came[t] > newest - recent else -(float(now[t]) if now[t] > 0 else 0.0), t))
            stays = set(order[:keep])
            dst = [t for t in range(keep) if t not in stays]
            src = [t for t in range(keep, L) if t in stays]
            assert len(src) == len(dst)
            now[dst], came[dst] = now[src], came[src]
            r["weights"][b, g, :keep], r["positions"][b, g, :keep] = now[:keep], came[:keep]
            _move(w, r, b, g, src, dst, keep)
    return r
