"""A round of a serving loop: prompts into the cache, their attention, alternatives from the logits, a tree of them verified, its best path committed, what the
budget does not hold evicted; against the same text recomputed in float64."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V, HIDDEN, HQ, HKV, D, P = 300, 48, 4, 2, 64, 16
SINKS, RECENT = 2, 8


class Model:
    """One attention layer between an embedding and a head, weights in float64."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.embedding = rng.standard_normal((V, HIDDEN))
        self.qkv = rng.standard_normal((HIDDEN, (HQ + 2 * HKV) * D)) * 2 / np.sqrt(HIDDEN)
        self.head = rng.standard_normal((HQ * D, V)) * 3 / np.sqrt(HQ * D)
        self.f = so.frequencies(D, 1e4)[0]

    def project(self, tokens):
        return (self.embedding[tokens] @ self.qkv).reshape(len(tokens), HQ + 2 * HKV, D)

    def logits(self, text, kept=None):
        """Of the text's last token.  kept [Hkv]: the places that each head still holds."""
        x = self.project(text)
        at = np.arange(len(text))
        q, k, v = so.rotate(x[:, :HQ], at, self.f), so.rotate(x[:, HQ:HQ + HKV], at, self.f), x[:, HQ + HKV:]
        out = np.zeros((HQ, D))
        for h in range(HQ):
            g = h // (HQ // HKV)
            seen = at if kept is None else np.asarray(kept[g])
            s = k[seen, g] @ q[-1, h] / np.sqrt(D)
            p = np.exp(s - s.max())
            out[h] = (p / p.sum()) @ v[seen, g]
        return out.reshape(-1) @ self.head


def test_a_round():
    model = Model(1)
    put = lambda x, t=torch.float32: torch.tensor(np.asarray(x), dtype=t, device=DEV)
    ints = lambda v: put(v, torch.int32)
    rng = np.random.default_rng(2)
    B, prompts = 3, [[int(t) for t in rng.integers(0, V, n)] for n in (37, 16, 61)]
    longest, pages = 96, 6
    kv = pa.KvCache(k_pool=torch.full((B * pages, HKV, P, D), float("nan"), device=DEV), v_pool=torch.full((B * pages, HKV, P, D), float("nan"), device=DEV),
                    block_table=ints(rng.permutation(B * pages).reshape(B, pages)), seq_lens=ints([len(p) for p in prompts]), num_q_heads=HQ, q_dtype="f32",
                    kv_dtype="f32", sm_scale=D ** -0.5, max_seq_len=longest)
    f, amplitude = pa.pillar_rope_frequencies(D, 1e4)
    rope = pa.Rope(f.to(DEV), False, amplitude)
    weights, positions = torch.zeros(B, HKV, longest, device=DEV), torch.zeros(B, HKV, longest, dtype=torch.int32, device=DEV)
    scores = torch.zeros(B, HKV, longest, device=DEV)
    head = put(model.head)

    def enter(tokens, starts, most, at=None):
        """New tokens' keys and values into the cache; their queries."""
        x = put(model.project(tokens))
        q = torch.empty(len(tokens), HQ, D, device=DEV)
        pa.pillar_append_rotated(kv, rope, x[:, HQ:HQ + HKV], x[:, HQ + HKV:], most, starts=ints(starts), positions=None if at is None else ints(at), q=x[:, :HQ], q_out=q)
        return q

    def look(logits, tokens=None, top=3):
        R = logits.shape[0]
        ids, lp = torch.zeros(R, top, dtype=torch.int32, device=DEV), torch.zeros(R, top, device=DEV)
        given = None if tokens is None else torch.zeros(R, tokens.shape[1], device=DEV)
        ws = torch.empty(pa.pillar_logprobs_workspace_bytes(R, V, top), dtype=torch.uint8, device=DEV)
        pa.pillar_token_logprobs(logits, ws, tokens=tokens, logprobs=given, top_ids=ids, top_logprobs=lp)
        return ids.cpu().numpy(), lp.cpu().numpy(), None if given is None else given.cpu().numpy()

    def soft(x):
        return x - x.max() - np.log(np.exp(x - x.max()).sum())

    # the prompts
    starts = [0, 37, 53, 114]
    q = enter([t for p in prompts for t in p], starts, 61)
    out = torch.empty_like(q)
    pa.pillar_prompt_attn(kv, q, 61, out, None, torch.empty(pa.pillar_prompt_workspace_bytes(kv, 114, 61), dtype=torch.uint8, device=DEV), starts=ints(starts))
    last = out[[36, 52, 113]].reshape(B, -1) @ head
    ids, lp, _ = look(last)
    texts = [list(p) for p in prompts]
    for b in range(B):
        want = model.logits(texts[b])
        assert ids[b].tolist() == np.argsort(-want, kind="stable")[:3].tolist()
        assert np.abs(lp[b] - np.sort(soft(want))[::-1][:3]).max() < 1e-3

    # a tree: the best token, then three others after it, then one after each of those; node i's place in the text goes by its depth
    parent, depth = [-1, 0, 0, 0, 1, 2, 3], [0, 1, 1, 1, 2, 2, 2]
    N = len(parent)
    words = []
    for i, p in enumerate(parent):
        words.append((words[p] if p >= 0 else 0) | 1 << i)
    tree = np.zeros((B, N), dtype=int)
    for b in range(B):
        best = int(ids[b, 0])
        after = np.argsort(-model.logits(texts[b] + [best]))[[0, 4, 9]]     # (one of the three is what the model says, in some place)
        after = np.roll(after, b)
        tree[b] = [best, *after, *[int(np.argsort(-model.logits(texts[b] + [best, int(t)]))[0]) for t in after]]
    before = [len(t) for t in texts]
    kv.seq_lens = ints([n + N for n in before])
    q = enter(tree.reshape(-1), [0, N, 2 * N, 3 * N], N, [before[b] + d for b in range(B) for d in depth])
    out, visible = torch.empty(B, N, HQ, D, device=DEV), put([words] * B, torch.int64)
    pa.pillar_verify_tree(kv, q.view(B, N, HQ, D), None, visible, out, None, scores, torch.empty(pa.pillar_tree_workspace_bytes(kv, N), dtype=torch.uint8, device=DEV))
    children = np.full((B, N, 3), -1)
    for i, p in enumerate(parent):
        if p >= 0:
            children[:, p, (children[0, p] >= 0).sum()] = tree[:, i]
    ids, _, given = look((out.reshape(B * N, -1) @ head), ints(children.reshape(B * N, 3)), 1)
    ids, given = ids.reshape(B, N), given.reshape(B, N, 3)
    for b in range(B):
        for i in range(N):
            path, at = [], i
            while at >= 0:
                path.insert(0, int(tree[b, at]))
                at = parent[at]
            want = model.logits(texts[b] + path)
            assert ids[b, i] == np.argmax(want), (b, i)
            for c, t in enumerate(children[b, i]):
                assert np.isneginf(given[b, i, c]) if t < 0 else abs(given[b, i, c] - soft(want)[t]) < 1e-3

    # accepted: from the root on, the child that the model itself says
    paths = []
    for b in range(B):
        path = [0]
        while True:
            hit = [i for i, p in enumerate(parent) if p == path[-1] and tree[b, i] == ids[b, path[-1]]]
            if not hit:
                break
            path += hit[:1]
        paths.append(path)
        assert len(path) == 3
        texts[b] += [int(tree[b, i]) for i in path]
    new_lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    pa.pillar_tree_commit(kv, None, N, ints(paths), ints([3] * B), new_lens, scores)
    assert new_lens.tolist() == [len(t) for t in texts]
    kv.seq_lens = new_lens.clone()

    # the budget: half of each context stays, the newest always among it
    budgets = [n // 2 for n in new_lens.tolist()]
    pa.pillar_evict_kv(kv, scores, 0.9, ints([0] * B), ints(budgets), SINKS, RECENT, weights, positions, new_lens,
                       torch.empty(pa.pillar_evict_workspace_bytes(kv), dtype=torch.uint8, device=DEV))
    kv.seq_lens = new_lens.clone()
    assert new_lens.tolist() == budgets

    # one more token each, as single rows of the prompt's call: its place in the text is not its number in the cache
    kv.seq_lens = ints([n + 1 for n in budgets])
    token = [int(ids[b, paths[b][-1]]) for b in range(B)]
    q = enter(token, [0, 1, 2, 3], 1, [len(t) for t in texts])
    out = torch.empty_like(q)
    pa.pillar_prompt_attn(kv, q, 1, out, None, torch.empty(pa.pillar_prompt_workspace_bytes(kv, B, 1), dtype=torch.uint8, device=DEV))
    ids, lp, _ = look(out.reshape(B, -1) @ head)
    places = positions.cpu().numpy()
    for b in range(B):
        texts[b].append(token[b])
        kept = [sorted(places[b, g, :budgets[b]].tolist()) + [len(texts[b]) - 1] for g in range(HKV)]
        assert all(len(set(k)) == budgets[b] + 1 for k in kept)
        want = model.logits(texts[b], kept)
        assert ids[b, 0] == np.argmax(want)
        assert np.abs(lp[b] - np.sort(soft(want))[::-1][:3]).max() < 1e-3


@pytest.mark.parametrize("kv_dtype", ["bf16", "fp8_e4m3"])
def test_a_prompt_in_chunks_is_the_prompt(kv_dtype):
    """Chunks appended and attended to one after the other, against the whole at once: with bf16 the cache has the same bits, with fp8 pages that grew
    over two chunks were rounded twice."""
    rng = np.random.default_rng(3)
    T, fp8 = 150, kv_dtype == "fp8_e4m3"
    rows = torch.from_numpy(rng.standard_normal((T, HQ + 2 * HKV, D)).astype(np.float32)).bfloat16().to(DEV)
    rope = pa.Rope(pa.pillar_rope_frequencies(D, 1e4)[0].to(DEV))

    def cache():
        pool = lambda: torch.zeros(12, HKV, P, D, dtype=torch.uint8 if fp8 else torch.bfloat16, device=DEV)
        scale = lambda: torch.ones(12, HKV, device=DEV) if fp8 else None
        return pa.KvCache(k_pool=pool(), v_pool=pool(), block_table=torch.arange(12, dtype=torch.int32, device=DEV)[None], seq_lens=torch.zeros(1, dtype=torch.int32, device=DEV),
                          num_q_heads=HQ, q_dtype="bf16", kv_dtype=kv_dtype, sm_scale=D ** -0.5, max_seq_len=T, k_scale=scale(), v_scale=scale())

    def fill(kv, cuts):
        outs, at = [], 0
        for n in cuts:
            kv.seq_lens.fill_(at + n)
            x, q = rows[at:at + n], torch.empty(n, HQ, D, dtype=torch.bfloat16, device=DEV)
            pa.pillar_append_rotated(kv, rope, x[:, HQ:HQ + HKV], x[:, HQ + HKV:], n, q=x[:, :HQ], q_out=q)
            outs.append(torch.empty_like(q))
            pa.pillar_prompt_attn(kv, q, n, outs[-1], None, torch.empty(pa.pillar_prompt_workspace_bytes(kv, n, n), dtype=torch.uint8, device=DEV))
            at += n
        return torch.cat(outs)

    whole, parts = cache(), cache()
    a, b = fill(whole, [T]), fill(parts, [1, 15, 16, 40, 77, 1])
    if not fp8:
        assert torch.equal(whole.k_pool, parts.k_pool) and torch.equal(whole.v_pool, parts.v_pool)
        # one definition, the same rounding of P and of the output: each is within 2^-8 of sum p |v| and of itself
        assert (a.double() - b.double()).abs().max() <= 4 * 2.0 ** -8 * rows[:, HQ + HKV:].abs().max()
    else:
        # a page's scale is the largest that its rows need, however they came; codes that were rounded twice are a step off at most
        assert torch.equal(whole.k_scale[:10], parts.k_scale[:10]) and torch.equal(whole.v_scale[:10], parts.v_scale[:10])
        f8 = lambda p: p.view(torch.float8_e4m3fn).float()
        for x, y in ((whole.k_pool, parts.k_pool), (whole.v_pool, parts.v_pool)):
            assert ((f8(x) - f8(y)).abs() <= 2.0 ** -3 * f8(x).abs() + 2.0 ** -9).all()


@pytest.mark.parametrize("kv_dtype", ["bf16", "fp8_e4m3"])
def test_pages_beyond_4_gib(kv_dtype):
    """The same request in the first pages of a small pool and in the last ones of a large one: the same bits."""
    fp8 = kv_dtype == "fp8_e4m3"
    rng = np.random.default_rng(4)
    T, heads, page = 300, 8, 256
    rows = torch.from_numpy(rng.standard_normal((T, 2 * heads + heads, 128)).astype(np.float32)).bfloat16().to(DEV)
    rope = pa.Rope(pa.pillar_rope_frequencies(128, 1e4)[0].to(DEV))

    def run(pages):
        pool = lambda: torch.zeros(pages, heads, page, 128, dtype=torch.uint8 if fp8 else torch.bfloat16, device=DEV)
        scale = lambda: torch.zeros(pages, heads, device=DEV) if fp8 else None
        kv = pa.KvCache(k_pool=pool(), v_pool=pool(), block_table=torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=DEV),
                        seq_lens=torch.tensor([T], dtype=torch.int32, device=DEV), num_q_heads=heads, q_dtype="bf16", kv_dtype=kv_dtype, sm_scale=128 ** -0.5,
                        max_seq_len=T, k_scale=scale(), v_scale=scale())
        q = torch.empty(T, heads, 128, dtype=torch.bfloat16, device=DEV)
        pa.pillar_append_rotated(kv, rope, rows[:, heads:2 * heads], rows[:, 2 * heads:], T, q=rows[:, :heads], q_out=q)
        out, lse = torch.empty_like(q), torch.empty(T, heads, device=DEV)
        pa.pillar_prompt_attn(kv, q, T, out, lse, torch.empty(pa.pillar_prompt_workspace_bytes(kv, T, T), dtype=torch.uint8, device=DEV))
        return q, out, lse, kv.k_pool[[pages - 1, pages - 2]].clone(), kv.v_pool[[pages - 1, pages - 2]].clone()

    small, large = run(2), run((5 << 30) // (heads * page * 128 * (1 if fp8 else 2)))
    assert all(torch.equal(a, b) for a, b in zip(small, large))
    assert small[1].isfinite().all() and (small[3].view(torch.float8_e4m3fn).float() if fp8 else small[3]).abs().max() > 0
