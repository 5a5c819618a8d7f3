"""The operators around a paged cache that a serving loop calls before and after its attention, over the shapes it gives them.

  rotate    rotary positions of queries (or keys) by themselves (`pillar_rotate`)
  append    queries and keys rotated, keys and values written into the paged cache (`pillar_append_rotated`)
  prompt    causal attention of new tokens, one or thousands per request, over the paged cache (`pillar_prompt_attn`)
  logprobs  log probabilities of given tokens, entropy and top alternatives of rows of logits (`pillar_token_logprobs`)

A case is one dict of plain values; `prepare` makes what the loop has in hand, `run` makes one pass, `exact` is the same from the
definitions in float64, request by request.
"""
from __future__ import annotations

import math
import random

import torch

own = False                # True: the package's operators; False: the same in elementary torch operations

DEVICE = "cuda:0"
SINKS = 4                  # first positions of a context: every query leans towards them
SHARED = 0.7               # weight of the direction that the queries of a KV head share
BASE = 1.0e6               # of the rotary frequencies

LAYER = dict(hq=32, hkv=8, dim=128, page=16, q="bf16", kv="bf16")           # attention layer of an 8B model


def listed():
    return [
        # the smallest rotation: eight tokens of a small fp32 layer, half of each head, neighbouring pairs
        dict(name="rotate_f32_t8", op="rotate", tokens=8, heads=4, dim=64, q="f32", rotary=32, interleaved=True, scaling="none", far=512),
        # queries of a 32 K chunk far into a long text, frequencies scaled for it
        dict(name="rotate_t32k", op="rotate", tokens=32768, heads=32, dim=128, q="bf16", rotary=128, interleaved=False, scaling="ramp", far=131072),
        # one user, one token of plain decoding: launch and latency
        dict(LAYER, name="append_b1", op="append", batch=1, new=1, spread="equal", lo=2100, hi=2100, rotary=128, interleaved=False,
             scaling="none", far=0),
        # four whole prompts of 4 to 8 K tokens
        dict(LAYER, name="append_prompt_b4_8k", op="append", batch=4, new=8192, spread="half", lo=0, hi=0, rotary=128, interleaved=False,
             scaling="ramp", far=0),
        # a server's verification step on an fp8 cache: five new tokens for each of 64 requests, pages with older rows in them
        dict(LAYER, name="append_fp8_b64", op="append", batch=64, hq=64, kv="fp8_e4m3", new=5, spread="equal", lo=512, hi=8192, rotary=128,
             interleaved=False, scaling="bands", far=0),
        # two short prompts of a small fp32 layer behind a shared beginning
        dict(name="prompt_f32_b2", op="prompt", batch=2, hq=4, hkv=1, dim=64, page=16, q="f32", kv="f32", new=200, spread="half", lo=100, hi=300),
        # four whole prompts of 8 K tokens: the most arithmetic
        dict(LAYER, name="prompt_b4_8k", op="prompt", batch=4, new=8192, spread="equal", lo=0, hi=0),
        # a chunk of 1000 tokens of one prompt beside 31 requests that decode a token each
        dict(LAYER, name="prompt_mixed_b32", op="prompt", batch=32, new=1000, spread="one", lo=1024, hi=8192),
        # prompts of very unequal length over an fp8 cache that holds what came before
        dict(LAYER, name="prompt_fp8_b8", op="prompt", batch=8, hq=64, kv="fp8_e4m3", new=4096, spread="log", lo=0, hi=2048),
        # one decoded token: its probability, and what else could have been
        dict(name="logprobs_b1", op="logprobs", rows=1, vocab=150000, type="bf16", tokens=1, top=8, masked=False),
        # a verification step of 128 requests with five positions each
        dict(name="logprobs_r640", op="logprobs", rows=640, vocab=150000, type="bf16", tokens=1, top=1, masked=False),
        # trees: 60 nodes of 4 requests, fp32 logits, four children each to look up, twenty to draft from, under a grammar's mask
        dict(name="logprobs_f32_r240", op="logprobs", rows=240, vocab=50001, type="f32", tokens=4, top=20, masked=True),
    ]


# a drawn case costs no more than the largest listed ones: pairs of queries and tokens over all heads, elements, bytes of the cache
_MOST_PAIRS, _MOST_ELEMENTS, _MOST_BYTES = 4 * 32 * 8192 * 8192, 1.3e8, 2.0e9


def draw(rng):
    """One more case: 1 to 128 requests, 1 to 8 K new tokens after none to 32 K, any cache type; vocabularies of 1 to 200 K."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    c = dict(op=rng.choice(["rotate", "append", "append", "prompt", "prompt", "logprobs", "logprobs"]))
    if c["op"] == "logprobs":
        c["type"] = rng.choice(["bf16", "bf16", "f32"])
        c["vocab"] = log(1000, 200000)
        c["rows"] = max(1, min(log(1, 1000), int(0.75 * _MOST_ELEMENTS / c["vocab"])))
        c["tokens"] = rng.choice([0, 1, 1, rng.randint(2, 8)])
        c["top"] = rng.choice([0, 1, rng.randint(2, 8), rng.randint(9, 64)])
        c["masked"] = rng.random() < 0.3
        return c
    c["dim"] = rng.choice([64, 128, 128])
    if c["op"] != "prompt":
        c["rotary"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 2 * rng.randint(1, c["dim"] // 2)])
        c["interleaved"] = rng.random() < 0.4
        c["scaling"] = rng.choice(["none", "linear", "base", "ramp", "bands"])
        c["far"] = rng.choice([0, log(1000, 1000000)])
    if c["op"] == "rotate":
        c["q"] = rng.choice(["bf16", "bf16", "f32"])
        c["heads"] = rng.choice([1, 4, 8, 14, 32, 64])
        c["far"] = max(c["far"], 4096)
        c["tokens"] = min(log(1, 32768), int(_MOST_ELEMENTS / (c["heads"] * c["dim"])))
        return c
    c["kv"] = rng.choice(["bf16", "bf16", "fp8_e4m3", "f32"])
    c["q"] = "f32" if c["kv"] == "f32" else "bf16"
    c["page"] = rng.choice([1, 16, 16, 32, 64, 128])
    c["hkv"] = rng.choice([1, 2, 4, 8, 8])
    c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 4, 5, 8, 16])
    c["batch"] = log(1, 128)
    c["new"] = rng.choice([1, rng.randint(2, 16), log(16, 8192), log(64, 4096)])
    c["spread"] = rng.choice(["equal", "half", "log", "one"])
    c["hi"] = rng.choice([0, log(16, 32768)])
    c["lo"] = int(c["hi"] * rng.uniform(0.1, 1.0))
    longest = c["hi"] + c["new"]
    held = longest * c["hkv"] * 2 * c["dim"] * {"f32": 4, "bf16": 2, "fp8_e4m3": 1}[c["kv"]]
    if c["op"] == "prompt":                                # (fp32 products run at a sixteenth of the rate)
        pairs = c["new"] * longest * c["hq"] * (16 if c["kv"] == "f32" else 1)
        if pairs > _MOST_PAIRS:                            # one request alone is too much: fewer heads, then fewer tokens
            c["hq"] = c["hkv"] = 1
            c["new"] = max(1, min(c["new"], int(_MOST_PAIRS / (longest * (16 if c["kv"] == "f32" else 1)))))
            pairs = c["new"] * longest * (16 if c["kv"] == "f32" else 1)
        c["batch"] = max(1, min(c["batch"], int(_MOST_PAIRS / pairs)))
    else:
        c["batch"] = max(1, min(c["batch"], int(1.5e8 / (c["new"] * (c["hq"] + 2 * c["hkv"]) * c["dim"]))))
    c["batch"] = max(1, min(c["batch"], int(_MOST_BYTES / held)))
    return c


# ---------------------------------------------------------------- sizes ----
def _new_tokens(case):
    rng = random.Random(2512 + case["batch"])
    n = case["new"]
    one = {
        "equal": lambda b: n,
        "half": lambda b: rng.randint((n + 1) // 2, n),
        "log": lambda b: int(round(math.exp(rng.uniform(0.0, math.log(n))))),
        "one": lambda b: n if b == case["batch"] // 2 else 1,
    }[case["spread"]]
    return [one(b) for b in range(case["batch"])]


def _before(case):
    rng = random.Random(1278 + case["batch"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


_SIZE = {"f32": 4, "bf16": 2, "fp8_e4m3": 1}


def work(case):
    if case["op"] == "logprobs":
        outputs = 4 * (2 * case["tokens"] + 2 + 2 * case["top"])
        return {"bytes": case["rows"] * (case["vocab"] * _SIZE[case["type"]] + outputs), "flops": 6 * case["rows"] * case["vocab"]}
    if case["op"] == "rotate":
        elements = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * elements * _SIZE[case["q"]] + 4 * case["tokens"] + 4 * case["rotary"],
                "flops": 3 * case["tokens"] * case["heads"] * case["rotary"]}
    kv, qo = _SIZE[case["kv"]], _SIZE[case["q"]]
    hq, hkv, d, page = case["hq"], case["hkv"], case["dim"], case["page"]
    total = {"bytes": 0, "flops": 0}
    for n, before in zip(_new_tokens(case), _before(case)):
        if case["op"] == "append":
            pages = (before + n - 1) // page - before // page + 1
            total["bytes"] += n * (2 * hq + 2 * hkv) * d * qo + 2 * n * hkv * d * kv + 4 * pages + 8 + (4 * n if case["far"] else 0)
            if case["kv"] == "fp8_e4m3":
                total["bytes"] += 8 * hkv * (pages + (before % page != 0))
            total["flops"] += 3 * n * (hq + hkv) * case["rotary"]
        else:
            total["bytes"] += n * hq * (2 * d * qo + 4) + 2 * (before + n) * hkv * d * kv + 4 * -(-(before + n) // page) + 8
            if case["kv"] == "fp8_e4m3":
                total["bytes"] += 8 * hkv * -(-(before + n) // page)
            total["flops"] += 4 * hq * d * (n * before + n * (n + 1) // 2)
    return total


# --------------------------------------------------------------- inputs ----
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _frequencies(case):
    """Angle per position of every pair, in 64 bits, and the factor on rotated pairs: the formulas of long-context scalings.
    Contexts of `trained` positions are stretched by `factor`."""
    r, factor, trained = case["rotary"], 4.0, 32768.0
    i = torch.arange(r // 2, dtype=torch.float64)
    f = BASE ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "base":
        return (BASE * factor ** (r / max(r - 2, 1))) ** (-2.0 * i / r), 1.0
    turns = trained * f / (2.0 * math.pi)
    if case["scaling"] == "ramp":                           # from pairs of 32 turns and more, unchanged, to those of one, stretched
        at = lambda n: r * math.log(trained / (2.0 * math.pi * n)) / (2.0 * math.log(BASE))
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        share = ((i - low) / max(high - low, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - share) + f / factor * share, 0.1 * math.log(factor) + 1.0
    if case["scaling"] == "bands":                          # from four turns, unchanged, to one, stretched
        share = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        return f * (share + (1.0 - share) / factor), 1.0
    return f, 1.0


def _scaling(case):
    """The same, as the package names it."""
    fast, slow = {"ramp": (32.0, 1.0), "bands": (4.0, 1.0)}.get(case["scaling"], (0.0, 0.0))
    return dict(scaling=case["scaling"], factor=4.0, original_len=32768, fast=fast, slow=slow)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    randn = lambda *shape, **kw: torch.randn(*shape, generator=gen, device=DEVICE, **kw)
    as_int = lambda v: torch.tensor(v, dtype=torch.int32, device=DEVICE)
    empty = lambda *shape: torch.zeros(*shape, device=DEVICE)
    s = dict(op=case["op"])
    if own:
        import paper_2512_01278_amd as pa
        s["pa"] = pa

    if case["op"] == "logprobs":
        R, V, M, N = case["rows"], case["vocab"], case["tokens"], case["top"]
        x = randn(R, V).mul_(2.5)
        likely = torch.randint(0, V, (R, 16), generator=gen, device=DEVICE)
        x.scatter_add_(1, likely, 9.0 + 2.0 * randn(R, 16))                 # a few tokens share most of the probability
        if case["masked"]:
            x.masked_fill_(torch.rand(R, V, generator=gen, device=DEVICE) < 0.9, -math.inf)
        s["logits"] = x.to(_DTYPE[case["type"]])
        drafted = torch.randint(0, V, (R, M), generator=gen, device=DEVICE)
        pick = torch.randint(0, 16, (R, M), generator=gen, device=DEVICE)
        s["tokens"] = torch.where(torch.rand(R, M, generator=gen, device=DEVICE) < 0.7, likely.gather(1, pick), drafted).to(torch.int32) if M else None
        s["scale"] = 1.0 / 0.8                                              # of a temperature
        s["logprobs"] = empty(R, M) if M else None
        s["lse"], s["entropy"] = empty(R), empty(R)
        s["top_ids"] = torch.zeros(R, N, dtype=torch.int32, device=DEVICE) if N else None
        s["top_logprobs"] = empty(R, N) if N else None
        if own:
            s["workspace"] = torch.empty(pa.pillar_logprobs_workspace_bytes(R, V, N), dtype=torch.uint8, device=DEVICE)
        return s

    qt, d = _DTYPE[case["q"]], case["dim"]
    if case["op"] != "prompt":
        f, amplitude = _frequencies(case)
        s["frequencies"], s["amplitude"], s["interleaved"] = f.to(DEVICE), amplitude, case["interleaved"]
        if own:
            mine, amplitude = pa.pillar_rope_frequencies(case["rotary"], BASE, **_scaling(case))
            s["rope"] = pa.Rope(mine.to(DEVICE), case["interleaved"], amplitude)
    if case["op"] == "rotate":
        T = case["tokens"]
        s["x"] = randn(T, case["heads"], d, dtype=qt)
        first = rng.randint(0, case["far"])
        s["positions"] = as_int(range(first, first + T))
        s["out"] = torch.zeros(T, case["heads"], d, dtype=qt, device=DEVICE)
        return s

    # a cache whose pool holds a quarter more pages than the batch needs, in no order
    new, before = _new_tokens(case), _before(case)
    B, hq, hkv, page = case["batch"], case["hq"], case["hkv"], case["page"]
    lens = [n + m for n, m in zip(new, before)]
    per = [-(-n // page) for n in lens]
    pages = sum(per) + -(-sum(per) // 4)
    order = torch.randperm(pages, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros(B, max(per), dtype=torch.int32, device=DEVICE)
    at = 0
    for b in range(B):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
    wide = torch.bfloat16 if case["kv"] == "bf16" else torch.float32
    k_pool = randn(pages, hkv, page, d, dtype=wide)
    v_pool = randn(pages, hkv, page, d, dtype=wide)
    base = randn(B, hkv, d)
    for t in range(min(SINKS, min(lens))):                                  # attention sinks
        k_pool[table[:, t // page].long(), :, t % page] += (10.0 * base / math.sqrt(d)).to(wide)
    k_scale = v_scale = None
    if case["kv"] == "fp8_e4m3":                                            # one scale per page and KV head
        # (tokens of some pages are larger than others', as activations are)
        k_pool *= 2.0 ** torch.randint(-1, 2, (pages, hkv, 1, 1), generator=gen, device=DEVICE)
        v_pool *= 2.0 ** torch.randint(-1, 2, (pages, hkv, 1, 1), generator=gen, device=DEVICE)

        def quantise(pool):
            scale = pool.abs().amax(dim=(2, 3)) / 448.0
            return (pool / scale[:, :, None, None]).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale
        k_pool, k_scale = quantise(k_pool)
        v_pool, v_scale = quantise(v_pool)
    T = sum(new)
    ends = [sum(new[:b]) for b in range(B + 1)]
    s.update(k_pool=k_pool, v_pool=v_pool, k_scale=k_scale, v_scale=v_scale, table=table, lens=as_int(lens), starts=as_int(ends), page=page,
             sm_scale=1.0 / math.sqrt(d), hq=hq, hkv=hkv, dim=d, widest=max(lens), most=max(new))
    s["request"] = torch.repeat_interleave(torch.arange(B, device=DEVICE), as_int(new).long())
    s["slot"] = torch.arange(T, device=DEVICE) + (s["lens"] - s["starts"][1:])[s["request"]].long()
    if own:
        s["kv"] = pa.KvCache(k_pool=k_pool, v_pool=v_pool, block_table=table, seq_lens=s["lens"], num_q_heads=hq, q_dtype=case["q"],
                             kv_dtype=case["kv"], sm_scale=s["sm_scale"], max_seq_len=max(lens), k_scale=k_scale, v_scale=v_scale)
    if case["op"] == "append":
        fused = randn(T, hq + 2 * hkv, d, dtype=qt)                         # what one projection gives for a token
        s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        s["q_out"] = torch.zeros(T, hq, d, dtype=qt, device=DEVICE)
        # after evictions the place in the text is not the slot
        s["positions"] = (s["slot"] + rng.randint(0, case["far"])).to(torch.int32) if case["far"] else None
    else:
        lean = SHARED * base[s["request"]][:, :, None, :]
        s["q"] = (lean + math.sqrt(1 - SHARED ** 2) * randn(T, hkv, hq // hkv, d)).reshape(T, hq, d).to(qt)
        s["out"] = torch.zeros(T, hq, d, dtype=qt, device=DEVICE)
        s["lse"] = empty(T, hq)
        if own:
            s["workspace"] = torch.empty(pa.pillar_prompt_workspace_bytes(s["kv"], T, s["most"]), dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------- one pass ----
def _pools(s):
    """The cache after a pass: 8-bit codes as the numbers they stand for, beside their scales."""
    if s["k_scale"] is None:
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    f8 = torch.float8_e4m3fn
    return {"k_pool": s["k_pool"].view(f8), "v_pool": s["v_pool"].view(f8), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def run(s):
    if s["op"] == "rotate":
        if own:
            s["pa"].pillar_rotate(s["x"], s["positions"], s["rope"], s["out"])
        else:
            s["out"].copy_(_rotated(s, s["x"], s["positions"]))
        return {"out": s["out"]}
    if s["op"] == "append":
        if own:
            s["pa"].pillar_append_rotated(s["kv"], s["rope"], s["k"], s["v"], s["most"], starts=s["starts"], positions=s["positions"],
                                          q=s["q"], q_out=s["q_out"])
        else:
            _append(s)
        return dict(_pools(s), q_out=s["q_out"])
    if s["op"] == "prompt":
        if own:
            s["pa"].pillar_prompt_attn(s["kv"], s["q"], s["most"], s["out"], s["lse"], s["workspace"], starts=s["starts"])
        else:
            _prompt(s)
        return {"out": s["out"], "lse": s["lse"]}
    if own:
        s["pa"].pillar_token_logprobs(s["logits"], s["workspace"], tokens=s["tokens"], logprobs=s["logprobs"], lse=s["lse"], entropy=s["entropy"],
                                      top_ids=s["top_ids"], top_logprobs=s["top_logprobs"], scale=s["scale"])
    else:
        _logprobs(s)
    return {k: s[k] for k in ("logprobs", "lse", "entropy", "top_ids", "top_logprobs") if s[k] is not None}


# ---------------------------------- the plain forms: elementary operations ----
def _pairs(s, x):
    """The two halves of every pair, and what is not rotated."""
    r = 2 * s["frequencies"].numel()
    if s["interleaved"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _rotated(s, x, positions):
    """[T, H, D] in fp32; angles in 64 bits."""
    x = x.float()
    turn = positions.double()[:, None, None] * s["frequencies"]
    cos, sin = (turn.cos() * s["amplitude"]).float(), (turn.sin() * s["amplitude"]).float()
    a, b, rest = _pairs(s, x)
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([a, b], dim=-1).flatten(-2) if s["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([both, rest], dim=-1)


def _append(s):
    positions = s["slot"] if s["positions"] is None else s["positions"]
    s["q_out"].copy_(_rotated(s, s["q"], positions))
    page, table = s["page"], s["table"].long()
    number = s["slot"] // page
    pid, slot = table[s["request"], number], s["slot"] % page
    for name, x in (("k", _rotated(s, s["k"], positions)), ("v", s["v"].float())):
        pool, scale = s[name + "_pool"], s[name + "_scale"]
        if scale is None:
            pool[pid, :, slot] = x.to(pool.dtype)
            continue
        # a page takes the larger of what its older rows had (where there are any) and what the new ones need; older rows are rounded anew
        cells = table.shape[0] * table.shape[1]
        cell = s["request"] * table.shape[1] + number
        most = torch.full((cells, s["hkv"]), -1.0, device=DEVICE)
        most.scatter_reduce_(0, cell[:, None].expand(-1, s["hkv"]), x.abs().amax(dim=2), "amax")
        touched = (most[:, 0] >= 0).nonzero()[:, 0]
        at = table.flatten()[touched]
        first = (s["lens"] - (s["starts"][1:] - s["starts"][:-1])).long()[touched // table.shape[1]]
        older = (first - touched % table.shape[1] * page).clamp(0, page)                          # older rows of the page
        had, fresh = scale[at], most[touched] / 448.0
        now = torch.where(older[:, None] > 0, torch.maximum(had, fresh), fresh)
        ratio = torch.where(had == now, 1.0, had / now)
        whole = pool[at].view(torch.float8_e4m3fn).float()                                        # [pages, Hkv, P, D]
        stays = torch.arange(page, device=DEVICE)[None, :] < older[:, None]
        whole = torch.where(stays[:, None, :, None], whole * ratio[:, :, None, None], whole)
        pool[at] = whole.to(torch.float8_e4m3fn).view(torch.uint8)
        scale[at] = now
        codes = (x * (1.0 / scale[pid])[:, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        pool[pid, :, slot] = codes.view(torch.uint8)


def _context(s, pool, scale):
    """[B, Hkv, T, D] in fp32: the rows of every request in order, T whole pages."""
    x = (pool if scale is None else pool.view(torch.float8_e4m3fn))[s["table"].long()].float()        # [B, pages, Hkv, P, D]
    if scale is not None:
        x = x * scale[s["table"].long()][:, :, :, None, None]
    return x.transpose(1, 2).reshape(x.shape[0], s["hkv"], -1, s["dim"])


def _prompt(s):
    B, hkv, hq, d, N = s["table"].shape[0], s["hkv"], s["hq"], s["dim"], s["most"]
    group = hq // hkv
    k, v = _context(s, s["k_pool"], s["k_scale"]), _context(s, s["v_pool"], s["v_scale"])
    T = k.shape[2]
    i = torch.arange(s["q"].shape[0], device=DEVICE) - s["starts"].long()[s["request"]]
    q = torch.zeros(B, N, hkv, group, d, device=DEVICE)
    q[s["request"], i] = s["q"].float().reshape(-1, hkv, group, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, hkv, N * group, d)
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["sm_scale"])
    first = (s["lens"] - (s["starts"][1:] - s["starts"][:-1])).long()
    last = first[:, None] + torch.arange(N, device=DEVICE)                                        # [B, N]: the last token a row sees
    hidden = torch.arange(T, device=DEVICE) > last.repeat_interleave(group, dim=1)[:, None, :, None]
    logits.masked_fill_(hidden, -math.inf)
    top = logits.amax(dim=3, keepdim=True)
    p = logits.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    out = torch.matmul(p.div_(total), v).reshape(B, hkv, N, group, d).permute(0, 2, 1, 3, 4).reshape(B, N, hq, d)
    lse = (top + total.log()).reshape(B, hkv, N, group).permute(0, 2, 1, 3).reshape(B, N, hq)
    s["out"].copy_(out[s["request"], i])
    s["lse"].copy_(lse[s["request"], i])


def _logprobs(s):
    x = s["logits"].float()
    z = x * s["scale"]
    top = z.amax(dim=1, keepdim=True)
    y = z - top
    e = y.exp()
    total = e.sum(dim=1, keepdim=True)
    lse = top + total.log()
    s["lse"].copy_(lse[:, 0])
    s["entropy"].copy_(total.log()[:, 0] - torch.where(e == 0, 0.0, e * y).sum(dim=1) / total[:, 0])
    if s["tokens"] is not None:
        s["logprobs"].copy_(z.gather(1, s["tokens"].long()) - lse)
    if s["top_ids"] is not None:
        # one whole number that grows with the logit and, among equal ones, towards the lower index
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -2147483648 - bits) * (1 << 24) - torch.arange(x.shape[1], device=DEVICE)
        ids = key.topk(s["top_ids"].shape[1], dim=1).indices
        s["top_ids"].copy_(ids)
        s["top_logprobs"].copy_(z.gather(1, ids) - lse)


# ----------------------------------------------------- the same in 64 bits ----
def exact(case, seed):
    s = prepare(case, seed)
    f64 = dict(dtype=torch.float64, device=DEVICE)
    if case["op"] == "logprobs":
        R = case["rows"]
        r = {k: torch.zeros(s[k].shape, **f64) for k in ("logprobs", "lse", "entropy", "top_logprobs") if s[k] is not None}
        if case["top"]:
            r["top_ids"] = torch.zeros(R, case["top"], dtype=torch.int32, device=DEVICE)
        for i in range(R):
            x = s["logits"][i].double() * s["scale"]
            p = torch.softmax(x, dim=0)
            r["lse"][i] = torch.logsumexp(x, dim=0)
            r["entropy"][i] = -torch.special.xlogy(p, p).sum()
            if case["tokens"]:
                r["logprobs"][i] = x[s["tokens"][i].long()] - r["lse"][i]
            if case["top"]:
                order = torch.sort(x, descending=True, stable=True).indices[:case["top"]]
                r["top_ids"][i], r["top_logprobs"][i] = order, x[order] - r["lse"][i]
        return {k: r[k] for k in ("logprobs", "lse", "entropy", "top_ids", "top_logprobs") if k in r}

    def turned(x, positions):
        """A pair as a complex number, times a unit one."""
        x = x.double()
        f, amplitude = _frequencies(case)
        m = f.numel()
        first = torch.arange(m, device=DEVICE) * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else m)
        unit = torch.polar(torch.full((x.shape[0], 1, m), amplitude, **f64), positions.double()[:, None, None] * f.to(DEVICE))
        y = torch.complex(x[..., first], x[..., second]) * unit
        x[..., first], x[..., second] = y.real.clone(), y.imag.clone()
        return x

    if case["op"] == "rotate":
        return {"out": turned(s["x"], s["positions"])}
    new, before, page, hkv = _new_tokens(case), _before(case), case["page"], case["hkv"]
    starts = s["starts"].tolist()
    if case["op"] == "append":
        r = {}
        place = torch.cat([torch.arange(m, m + n) for n, m in zip(new, before)]).to(DEVICE) if s["positions"] is None else s["positions"]
        for name, x in (("k", turned(s["k"], place)), ("v", s["v"].double())):
            pool, scale = s[name + "_pool"], s[name + "_scale"]
            if scale is None:
                r[name + "_pool"] = pool.double()
                for b, (n, m) in enumerate(zip(new, before)):
                    t = torch.arange(m, m + n, device=DEVICE)
                    r[name + "_pool"][s["table"][b, t // page].long(), :, t % page] = x[starts[b]:starts[b + 1]]
                continue
            # 8 bits: the scales have a value in 64 bits, the codes are what a rounding makes of it
            r[name + "_pool"], r[name + "_scale"] = None, scale.double()
            most = x.abs().amax(dim=2) / 448.0
            for b, (n, m) in enumerate(zip(new, before)):
                for p in range(m // page, (m + n - 1) // page + 1):
                    lo, hi = max(p * page - m, 0), min((p + 1) * page - m, n)
                    need = most[starts[b] + lo:starts[b] + hi].amax(dim=0)
                    id = int(s["table"][b, p])
                    r[name + "_scale"][id] = torch.maximum(r[name + "_scale"][id], need) if m > p * page else need
        r["q_out"] = turned(s["q"], place)
        return {k: r[k] for k in ("k_pool", "v_pool", "k_scale", "v_scale", "q_out") if k in r}
    r = {"out": torch.zeros(s["out"].shape, **f64), "lse": torch.zeros(s["lse"].shape, **f64)}
    group = case["hq"] // hkv
    for b, (n, m) in enumerate(zip(new, before)):
        ids = s["table"][b, :-(-(n + m) // page)].long()

        def rows(pool, scale):
            x = (pool if scale is None else pool.view(torch.float8_e4m3fn))[ids].double()
            if scale is not None:
                x = x * scale[ids].double()[:, :, None, None]
            return x.permute(1, 0, 2, 3).reshape(hkv, -1, case["dim"])[:, :n + m]

        k, v = rows(s["k_pool"], s["k_scale"]), rows(s["v_pool"], s["v_scale"])
        later = torch.arange(n + m, device=DEVICE)[None, :] > torch.arange(m, m + n, device=DEVICE)[:, None]
        mine = slice(starts[b], starts[b + 1])
        for h in range(case["hq"]):
            x = torch.matmul(s["q"][mine, h].double(), k[h // group].t().contiguous()) * s["sm_scale"]
            x.masked_fill_(later, -math.inf)
            lse = torch.logsumexp(x, dim=1)
            r["lse"][mine, h] = lse
            r["out"][mine, h] = torch.matmul(torch.exp(x - lse[:, None]), v[h // group])
    return r
