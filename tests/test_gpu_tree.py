"""Trees of drafted tokens on the GPU against the oracle: every kernel, head layout, page size and mask where they can go wrong."""
import dataclasses

import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2512_01278_amd as pa
from tests.tree_cases import TreeRun, ancestors, as_int64, cache_of, check_tree, make, queries

pytestmark = pytest.mark.gpu

GENERIC = pa.PILLAR_FLAG_GENERIC_KERNELS


def tree_case(what, lens, N, sizes=None, seed=1, flags=0, words=None, **shape):
    rng = np.random.default_rng(seed)
    w = make(what, seed, lens, **shape)
    if words is None:
        words = [ancestors(rng, N) for _ in lens]
    print(f"[case] {what}: lens={list(lens)[:6]} N={N} {shape}", flush=True)
    return TreeRun(w, N, sizes, words, seed=seed, flags=flags)


def verified(run, what):
    run.run()
    torch.cuda.synchronize()
    return check_tree(run, what)


SHAPES = [
    # rows per KV head: one to a wavefront's worth, two, four, eight, four times eight
    dict(Hq=8, Hkv=2, N=1), dict(Hq=8, Hkv=2, N=8), dict(Hq=8, Hkv=2, N=9), dict(Hq=8, Hkv=2, N=16), dict(Hq=8, Hkv=2, N=17), dict(Hq=4, Hkv=1, N=32),
    dict(Hq=4, Hkv=1, N=33), dict(Hq=4, Hkv=1, N=60), dict(Hq=16, Hkv=1, N=64), dict(Hq=3, Hkv=3, N=5), dict(Hq=14, Hkv=2, N=11),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s['Hq']}x{s['Hkv']}-{s['N']}")
@pytest.mark.parametrize("kv,D,flags", [("bf16", 128, 0), ("fp8_e4m3", 128, 0), ("bf16", 64, 0), ("fp8_e4m3", 64, 0), ("f32", 64, 0), ("bf16", 128, GENERIC)])
def test_rows_and_types(shape, kv, D, flags):
    N = shape["N"]
    run = tree_case(f"{kv}-{D}", [N, N + 1, 127 + N, 300, 64 + N], N, D=D, kv=kv, q="f32" if kv == "f32" else "bf16", flags=flags, Hq=shape["Hq"],
                    Hkv=shape["Hkv"], seed=N)
    verified(run, f"{shape} {kv} {D}")


@pytest.mark.parametrize("q,kv,D", [("f32", "f32", 128), ("f32", "bf16", 128), ("f32", "fp8_e4m3", 128), ("bf16", "f32", 128), ("f32", "bf16", 64),
                                    ("f32", "fp8_e4m3", 64), ("bf16", "f32", 64)])
def test_mixed_types(q, kv, D):
    for N, Hq in ((6, 4), (20, 8)):
        verified(tree_case(f"{q}/{kv}", [40, 201, N], N, q=q, kv=kv, D=D, Hq=Hq, Hkv=1, seed=N), f"{q} {kv} {D} {N}")


@pytest.mark.parametrize("P", [1, 2, 8, 16, 64, 256])
@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3", "f32"])
def test_page_sizes(P, kv):
    verified(tree_case(f"P{P}", [1, 63, 64, 65, 130, 257], 1, P=P, kv=kv, q="f32" if kv == "f32" else "bf16", seed=P), f"P={P} {kv} N=1")
    verified(tree_case(f"P{P}", [30, 64, 95, 96, 130, 257], 30, P=P, kv=kv, q="f32" if kv == "f32" else "bf16", seed=P), f"P={P} {kv} N=30")


@pytest.mark.parametrize("kv,flags", [("bf16", 0), ("fp8_e4m3", 0), ("bf16", GENERIC)])
def test_trees_of_different_sizes_and_of_none(kv, flags):
    run = tree_case("sizes", [50, 700, 9, 1, 333, 64, 0, 3], 24, sizes=[24, 1, 9, 1, 0, 17, 0, 3], kv=kv, flags=flags, seed=5)
    verified(run, "sizes")


@pytest.mark.parametrize("kv,flags", [("bf16", 0), ("fp8_e4m3", 0), ("f32", 0), ("bf16", GENERIC)])
def test_contexts_shorter_than_their_tree_and_rows_that_see_nothing(kv, flags):
    N = 12
    words = [[0] * N, [1 << i for i in range(N)], [0 if i % 3 else 2 ** (i + 1) - 1 for i in range(N)], [2 ** 64 - 1] * N, [1 << 11] * N, [2 ** 63] * N]
    run = tree_case("nothing", [N, N, 5, 7, 40, 1], N, words=words, kv=kv, q="f32" if kv == "f32" else "bf16", flags=flags, seed=6)
    verified(run, "nothing")
    assert not run.out[0].any() and torch.isneginf(run.lse[0]).all() and not run.scores[0, :, :N].any()


def test_an_empty_context_gives_zeros():
    run = tree_case("empty", [0, 20], 4, sizes=[4, 4], words=[[1, 3, 7, 15]] * 2)
    run.run()
    torch.cuda.synchronize()
    assert not run.out[0].any() and torch.isneginf(run.lse[0]).all() and torch.isnan(run.scores[0]).all()


@pytest.mark.parametrize("kv,flags", [("bf16", 0), ("fp8_e4m3", 0), ("f32", 0), ("bf16", GENERIC)])
@pytest.mark.parametrize("N", [7, 40])
def test_what_is_not_seen_has_no_influence(kv, flags, N):
    """Infinities and NaN in K and V of nodes: only the rows that see them may show them, and those do."""
    lens = [N, N + 50, 200]
    q = "f32" if kv == "f32" else "bf16"
    clean = tree_case("clean", lens, N, kv=kv, q=q, flags=flags, seed=8)
    # the last three nodes are seen by themselves only; the one before by nobody
    for b in range(3):
        for i in range(N):
            word = clean.words[b][i] & ~(15 << (N - 4))
            clean.words[b][i] = word | (1 << i if i >= N - 3 else 0)
    clean.visible = as_int64(clean.words).to(clean.visible.device)
    clean.run()
    w = clean.w
    bits = {"f32": [np.float32(np.inf), np.float32(np.nan)], "bf16": [np.uint16(0x7f80), np.uint16(0xffc0)], "fp8_e4m3": [np.uint8(0x7f), np.uint8(0xff)]}[kv]
    for b in range(3):
        for i, (pool, value) in ((N - 4, (w.k_pool, bits[1])), (N - 4, (w.v_pool, bits[1])), (N - 3, (w.v_pool, bits[0])), (N - 2, (w.k_pool, bits[1]))):
            t = lens[b] - N + i
            pool[w.block_table[b, t // w.P], :, t % w.P, ::3] = value
    dirty = TreeRun(w, N, None, clean.words, seed=8, flags=flags)
    dirty.run()
    torch.cuda.synchronize()
    assert torch.equal(dirty.out[:, :N - 3], clean.out[:, :N - 3]) and torch.equal(dirty.out[:, N - 1], clean.out[:, N - 1])
    assert torch.equal(dirty.lse[:, :N - 2], clean.lse[:, :N - 2]) and torch.equal(dirty.lse[:, N - 1], clean.lse[:, N - 1])
    hit = dirty.out[:, N - 3].float()
    assert not torch.isfinite(hit[..., ::3]).any() and torch.equal(hit[..., 1::3], clean.out[:, N - 3].float()[..., 1::3])
    assert torch.isnan(dirty.out[:, N - 2].float()).all() and torch.isnan(dirty.lse[:, N - 2]).all()


@pytest.mark.parametrize("kv,flags", [("bf16", 0), ("fp8_e4m3", 0), ("f32", 0)])
def test_strided_pools(kv, flags):
    """Slots outermost, and pools whose rows are not multiples of 16 bytes apart (those run in fp32)."""
    q = "f32" if kv == "f32" else "bf16"
    for N in (4, 20):
        run = tree_case("strided", [45, 200], N, kv=kv, q=q, seed=9, Hq=8, Hkv=2)
        pages, Hkv, P, D = run.kv.k_pool.shape
        slot_major = lambda x: x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
        odd = lambda x: torch.nn.functional.pad(x, (1, 2))[..., 1:-2]
        for change in (slot_major, odd):
            k, v = run.kv.k_pool, run.kv.v_pool
            run.kv.k_pool, run.kv.v_pool = change(k), change(v)
            assert not run.kv.k_pool.is_contiguous()
            for t in (run.out, run.lse, run.scores):
                t.fill_(float("nan"))
            verified(run, f"strided {kv} {N}")
            run.kv.k_pool, run.kv.v_pool = k, v


def test_tensors_off_a_16_byte_boundary():
    run = tree_case("offset", [45, 200], 5, seed=9)
    whole = torch.full((run.out.numel() + 1,), float("nan"), dtype=run.out.dtype, device=run.out.device)
    run.out = whole[1:].view(run.out.shape)
    verified(run, "out off the boundary")
    whole = torch.zeros(run.q.numel() + 1, dtype=run.q.dtype, device=run.q.device)
    whole[1:] = run.q.reshape(-1)
    run.q = whole[1:].view(run.q.shape)
    verified(run, "q off the boundary")


@pytest.mark.parametrize("N,kv", [(1, "bf16"), (8, "bf16"), (16, "fp8_e4m3"), (25, "bf16"), (60, "fp8_e4m3")])
def test_contexts_cut_into_many_ranges(N, kv):
    """One long request beside short ones: partial results of many workgroups, tiles that begin and end inside a range."""
    verified(tree_case("long", [5000 + N, N, 700, 64 + N], N, kv=kv, Hq=4, Hkv=1, seed=N), f"long {N} {kv}")


@pytest.mark.parametrize("lens,sizes", [([20001], None), ([12345, 3, 0, 6400], None), ([9000, 8999, 64], [0, 5, 1])])
@pytest.mark.parametrize("N,kv", [(5, "bf16"), (40, "bf16"), (13, "fp8_e4m3")])
def test_ranges_of_several_units(lens, sizes, N, kv):
    """One KV head and few requests: a range is several units long, and a tile has partials of a dozen or more."""
    verified(tree_case("several", lens, N, kv=kv, Hq=4, Hkv=1, sizes=sizes, seed=N), f"several {lens} {N} {kv}")


@pytest.mark.parametrize("N", [1, 10, 40])
def test_more_requests_than_a_wavefront_has_lanes(N):
    rng = np.random.default_rng(N)
    lens = rng.integers(N, 90, size=150)
    sizes = rng.integers(0, N + 1, size=150)
    sizes[70:140] = 0                                        # a whole run of requests without nodes
    verified(tree_case("many", lens, N, sizes=sizes, Hq=4, Hkv=1, D=64, seed=N), f"many {N}")


def test_more_work_than_workgroups():
    """Ranges of several tiles that pass from one (request, head) to the next."""
    rng = np.random.default_rng(3)
    lens = rng.integers(20, 400, size=40)
    verified(tree_case("ranges", lens, 20, Hq=16, Hkv=8, seed=3, D=64), "ranges")
    verified(tree_case("ranges", lens, 6, Hq=32, Hkv=16, seed=3, D=64), "ranges")


def test_logits_far_apart():
    """Maxima that grow along the context by steps below and above what an accumulator is left unscaled for."""
    for gain in (0.3, 3.0, 40.0):
        w = make("ramp", 4, [400], Hq=4, Hkv=1)
        ramp = (np.arange(400) / 400 * gain).astype(np.float32)
        q = np.tile(np.ones(128, np.float32), (1, 10, 4, 1))
        for t in range(400):
            row = np.full(128, ramp[t], np.float32) + np.random.default_rng(t).standard_normal(128).astype(np.float32) * 0.1
            w.k_pool[w.block_table[0, t // 16], 0, t % 16] = gen.bf16_bits_from_f32(row)
        bits = gen.bf16_bits_from_f32(q)
        run = TreeRun(w, 10, None, [ancestors(np.random.default_rng(1), 10)],
                      queries_of=(torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16), gen.f32_from_bf16_bits(bits).astype(np.float64)))
        verified(run, f"ramp {gain}")


def test_the_weightiest_token_of_an_fp8_page_is_not_rounded():
    """Of one tile the largest p v_scale is 1 before it is rounded to bf16, so a row that one token dominates carries the output's own rounding only: each
    other token's share is off by 2^-8 of itself, all else is that of the fp32 logits and sums."""
    w = make("peaked", 21, [60, 33, 17], Hq=4, Hkv=1, D=64, kv="fp8_e4m3")
    q, q64 = queries(np.random.default_rng(21), w, 1)
    run = TreeRun(w, 1, None, [ancestors(np.random.default_rng(21), 1)] * 3, queries_of=(q * 8, q64 * 8))
    verified(run, "peaked")
    table, got = oracle.e4m3_table(), run.out.double().cpu().numpy()
    reach = np.nanmax(oracle.verify_tree(w, run.q64, run.sizes, run.words)["reach"])
    prob = (2 * w.D * reach + 100) * 2.0 ** -24
    peaked = 0
    for b, n in enumerate(w.seq_lens):
        page = lambda t: w.block_table[b][t // w.P]
        scales = np.array([w.v_scale[page(t), 0] for t in range(n)], dtype=np.float64)
        k = np.array([table[w.k_pool[page(t), 0, t % w.P]] * np.float64(w.k_scale[page(t), 0]) for t in range(n)])
        v = np.array([table[w.v_pool[page(t), 0, t % w.P]] for t in range(n)]) * scales[:, None]
        for h in range(4):
            x = k @ np.asarray(q64[b, 0, h] * 8, dtype=np.float64) * w.sm_scale
            p = np.exp(x - x.max())
            p /= p.sum()
            top = np.argmax(p * scales)
            rest = (p[:, None] * np.abs(v)).sum(0) - p[top] * np.abs(v[top])
            bound = 2.0 ** -8 * np.abs(p @ v) + 2.0 ** -8 * (1 + 2.0 ** -8) * rest + prob * (p @ np.abs(v))
            assert (np.abs(got[b, 0, h] - p @ v) <= bound).all(), (b, h)
            peaked += p[top] > 0.5
    print(f"[peaked] {peaked} of 12 rows", flush=True)


def test_optional_outputs_and_the_bits_of_the_others():
    run = tree_case("optional", [900, 33], 13, seed=11)
    run.run()
    torch.cuda.synchronize()
    first = run.out.clone(), run.lse.clone(), run.scores.clone()
    for lse, scores in ((False, True), (True, False), (False, False), (True, True)):
        for t in (run.out, run.lse, run.scores):
            t.fill_(float("nan"))
        run.run(with_lse=lse, with_scores=scores)
        torch.cuda.synchronize()
        assert torch.equal(run.out, first[0])
        assert torch.equal(run.lse, first[1]) if lse else torch.isnan(run.lse).all()
        assert torch.equal(run.scores.nan_to_num(-1), first[2].nan_to_num(-1)) if scores else torch.isnan(run.scores).all()


def test_a_chain_agrees_with_the_verification_of_chains():
    w = gen.make_custom(name="chain", seed=3, B=3, Hq=8, Hkv=2, D=128, P=16, spec_k=4, q_dtype="bf16", kv_dtype="bf16", seq_lens=[5, 333, 1700], budgets=[1] * 3)
    q = torch.from_numpy(w.q.view(np.int16)).view(torch.bfloat16)
    run = TreeRun(w, 5, None, [[2 ** (i + 1) - 1 for i in range(5)]] * 3, queries_of=(q, gen.f32_from_bf16_bits(w.q).astype(np.float64)))
    verified(run, "chain")
    out, lse = torch.empty_like(run.out), torch.empty_like(run.lse)
    ws = torch.empty(pa.pillar_workspace_bytes(run.kv, 4, 1), dtype=torch.uint8, device=out.device)
    pa.pillar_verify_attn(run.kv, run.q, 4, out, lse, None, ws)
    torch.cuda.synchronize()
    assert (run.lse - lse).abs().max() <= 2e-5 and (run.out.float() - out.float()).abs().max() <= 2e-2


def test_rows_past_32_bits():
    """A pool of 4.4 G elements: the pages in use lie at its end."""
    D, P, Hkv = 128, 64, 8
    pages = (2 ** 32 + 2 ** 27) // (D * P * Hkv)
    w = make("far", 2, [150, 700], Hq=16, Hkv=Hkv, P=P)
    run = TreeRun(w, 9, None, [ancestors(np.random.default_rng(b), 9) for b in range(2)])
    small = run.kv.k_pool.shape[0]
    k = torch.empty(pages, Hkv, P, D, dtype=torch.bfloat16, device="cuda:0")
    k[-small:] = run.kv.k_pool
    v = torch.empty_like(k)
    v[-small:] = run.kv.v_pool
    run.kv.k_pool, run.kv.v_pool = k, v
    run.kv.block_table += pages - small
    verified(run, "far")
    path, lens = torch.tensor([[1, 4, 7], [0, 8, 0]], dtype=torch.int32, device="cuda:0"), torch.tensor([3, 2], dtype=torch.int32, device="cuda:0")
    now = torch.zeros_like(lens)
    want = oracle.tree_commit(w, [9, 9], path.cpu().numpy(), [3, 2])
    pa.pillar_tree_commit(run.kv, None, 9, path, lens, now)
    torch.cuda.synchronize()
    assert np.array_equal(k[-small:].view(torch.int16).cpu().numpy().view(np.uint16), want["k_pool"])


@pytest.mark.parametrize("kv,D", [("bf16", 128), ("fp8_e4m3", 128), ("bf16", 64), ("fp8_e4m3", 64)])
@pytest.mark.parametrize("N", [3, 12, 30, 50])
def test_bounds_far_above_the_lengths(kv, D, N):
    """Kernels are chosen by max_seq_len: with one that would mean gigabytes, rows bypass the cache and 50 nodes run on eight wavefronts."""
    rng = np.random.default_rng(N)
    w = make("bound", N, [N, 700, 64 + N, 1300], Hq=32, Hkv=8, D=D, P=64, kv=kv, extra_table_cols=400)
    run = TreeRun(w, N, None, [ancestors(rng, N) for _ in range(4)], seed=N)
    run.kv.max_seq_len = w.block_table.shape[1] * 64
    run.scores = torch.full((4, 8, run.kv.max_seq_len), float("nan"), device=run.out.device)
    run.workspace = torch.empty(pa.pillar_tree_workspace_bytes(run.kv, N), dtype=torch.uint8, device=run.out.device)
    verified(run, f"bound {kv} {D} {N}")


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    runs = [tree_case("at once", [900, 300, 40], 9, seed=s) for s in (1, 2)]
    for r in runs:
        r.run()
    torch.cuda.synchronize()
    first = [(r.out.clone(), r.lse.clone()) for r in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for r, s in zip(runs, streams):
            r.run(stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(r.out, f[0]) and torch.equal(r.lse, f[1]) for r, f in zip(runs, first))


def test_one_workspace_for_two_graphs():
    """Captured calls leave nothing behind that the other could trip over."""
    runs = [tree_case("shared", [500, 80], 9, seed=1), tree_case("shared", [70, 900, 33], 17, seed=2, kv="fp8_e4m3")]
    ws = max((r.workspace for r in runs), key=lambda t: t.numel())
    graphs, first = [], []
    for r in runs:
        r.workspace = ws
        r.run()
        torch.cuda.synchronize()
        first.append((r.out.clone(), r.lse.clone(), r.scores.clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.run()
        graphs.append(g)
    for turn in range(3):
        for r, g, f in zip(runs, graphs, first):
            for t in (r.out, r.lse, r.scores):
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(r.out, f[0]) and torch.equal(r.lse, f[1]) and torch.equal(r.scores.nan_to_num(-1), f[2].nan_to_num(-1)), turn


def test_tensors_of_another_device_are_refused():
    run = tree_case("device", [40], 4)
    for name in ("q", "out", "visible", "workspace"):
        was = getattr(run, name)
        setattr(run, name, was.cpu())
        with pytest.raises(ValueError):
            run.run()
        setattr(run, name, was)
    kv, run.kv = run.kv, dataclasses.replace(run.kv, k_pool=run.kv.k_pool.cpu())
    with pytest.raises(ValueError):
        run.run()
    run.kv = kv
    path, lens, now = torch.zeros(1, 2, dtype=torch.int32, device="cuda:0"), torch.zeros(1, dtype=torch.int32, device="cuda:0"), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        pa.pillar_tree_commit(run.kv, None, 4, path, lens, now)


def test_streams_and_graphs():
    """Another stream than the current one; a captured call, replayed with eager work between, gives the bits of the eager call."""
    run = tree_case("graph", [800, 60, 9], 9, seed=12)
    run.run()
    torch.cuda.synchronize()
    first = run.out.clone(), run.lse.clone(), run.scores.clone()
    side = torch.cuda.Stream()
    run.out.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    run.run(stream=side)
    side.synchronize()
    assert torch.equal(run.out, first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.run()
    for turn in range(4):
        for t in (run.out, run.lse, run.scores):
            t.fill_(float("nan"))
        run.workspace.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(run.out, first[0]) and torch.equal(run.lse, first[1]) and torch.equal(run.scores.nan_to_num(-1), first[2].nan_to_num(-1)), turn


# ---------------------------------------------------------------- commit ----
def committed(w, N, sizes, path, lens, with_scores=True):
    kv = cache_of(w)
    dev = kv.k_pool.device
    scores = torch.rand(w.B, w.Hkv, kv.max_seq_len + 1, device=dev) if with_scores else None
    want = oracle.tree_commit(w, sizes, np.asarray(path), lens, None if scores is None else scores.cpu().numpy())
    as_int = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device=dev)
    now = torch.full((w.B,), -7, dtype=torch.int32, device=dev)
    pa.pillar_tree_commit(kv, as_int(sizes), N, as_int(path), as_int(lens), now, scores)
    torch.cuda.synchronize()
    check_cache(kv, want)
    assert now.tolist() == want["new_lens"].tolist()
    if scores is not None:
        assert np.array_equal(scores.cpu().numpy(), want["scores"])


def check_cache(kv, want):
    for name in ("k_pool", "v_pool"):
        got = getattr(kv, name)
        got = got.view(torch.int16).cpu().numpy().view(np.uint16) if got.dtype == torch.bfloat16 else got.cpu().numpy()
        assert np.array_equal(got.view(np.uint8), want[name].view(np.uint8)), name
    for name in ("k_scale", "v_scale"):
        if name in want:
            assert np.array_equal(getattr(kv, name).cpu().numpy(), want[name], equal_nan=True), name


@pytest.mark.parametrize("kv,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64), ("fp8_e4m3", 128), ("fp8_e4m3", 64)])
@pytest.mark.parametrize("P", [1, 4, 16, 64])
def test_commit(kv, D, P):
    N = 64
    rng = np.random.default_rng(P)
    lens, sizes = [64, 65, 300, 131, 40, 80], [64, 64, 50, 3, 40, 0]
    w = make("commit", P, lens, kv=kv, q="f32" if kv == "f32" else "bf16", D=D, P=P, Hq=4, Hkv=2)
    path = np.full((6, 64), -1)
    for b in range(6):
        if sizes[b]:
            path[b, :sizes[b]] = np.sort(rng.permutation(sizes[b]))
    counts = [64, 20, 50, 2, 0, 5]
    for b, keep in enumerate(counts):
        if 0 < keep < sizes[b]:
            path[b, :keep] = np.sort(rng.choice(sizes[b], keep, replace=False))
    committed(w, N, sizes, path, counts)
    # any order, the same node twice, entries that are no nodes, counts beyond the list
    path = rng.integers(0, 64, size=(6, 7))
    path[0, 3], path[1, 0], path[2, 6] = 64, -1, 1000
    committed(w, N, sizes, path, [7, 7, 9, 7, -3, 7], with_scores=False)


def test_commit_of_a_tree_that_is_not_in_the_cache():
    w = make("short", 1, [5, 9], Hq=4, Hkv=2)
    committed(w, 8, [8, 8], [[1, 2], [3, 4]], [2, 2])


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_commit_replayed(kv):
    w = make("replay", 3, [100, 37], kv=kv, Hq=4, Hkv=2)
    kv_ = cache_of(w)
    dev = kv_.k_pool.device
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    path, lens, now = ints([[1, 3, 4], [0, 2, 5]]), ints([3, 2]), ints([0, 0])
    before = kv_.k_pool.clone(), kv_.v_pool.clone(), None if kv_.k_scale is None else kv_.k_scale.clone(), None if kv_.v_scale is None else kv_.v_scale.clone()
    want = oracle.tree_commit(w, [6, 6], path.cpu().numpy(), [3, 2])
    pa.pillar_tree_commit(kv_, None, 6, path, lens, now)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.pillar_tree_commit(kv_, None, 6, path, lens, now)
    for _ in range(3):
        for t, old in zip((kv_.k_pool, kv_.v_pool, kv_.k_scale, kv_.v_scale), before):
            if t is not None:
                t.copy_(old)
        graph.replay()
        torch.cuda.synchronize()
        check_cache(kv_, want)
