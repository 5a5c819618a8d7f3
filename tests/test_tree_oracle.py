"""The oracle of trees and of the bounded cache, pinned by reduction to the chain's, by closed forms and by hand; and what the entry points
refuse, on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

import gen
import oracle
from paper_2512_01278_amd import binding as pb
from tests.test_abi import FAKE, good_kv, lib  # noqa: F401  (a fixture)
from tests.tree_cases import ancestors, as_int64, make


def test_a_chain_is_what_verification_computes():
    w = gen.make_custom(name="chain", seed=3, B=3, Hq=4, Hkv=2, D=64, P=16, spec_k=4, q_dtype="f32", kv_dtype="f32", seq_lens=[5, 33, 70], budgets=[1] * 3)
    want = oracle.verify_attn(w)
    got = oracle.verify_tree(w, w.q.astype(np.float64), [5] * 3, [[2 ** (i + 1) - 1 for i in range(5)]] * 3)
    np.testing.assert_allclose(got["out"], want[0], rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(got["lse"], want[1], rtol=1e-12)
    for b in range(3):
        n = w.seq_lens[b]
        np.testing.assert_allclose(got["scores"][b, :, :n], want[2][b, :, :n], rtol=1e-12, atol=1e-15)


def test_a_path_of_a_tree_is_a_chain_of_its_own():
    """What a node sees is what it would see had only its ancestors been drafted."""
    rng = np.random.default_rng(5)
    w = make("path", 7, [40], Hq=2, Hkv=1, D=64, q="f32", kv="f32", P=1)
    n = 9
    words = ancestors(rng, n)
    q = rng.standard_normal((1, n, 2, 64))
    tree = oracle.verify_tree(w, q, [n], [words])
    for i in range(n):
        line = [j for j in range(n) if words[i] >> j & 1]
        short = make("path", 7, [40], Hq=2, Hkv=1, D=64, q="f32", kv="f32", P=1)
        first = 40 - n
        short.block_table[0, :first + len(line)] = np.concatenate([w.block_table[0, :first], w.block_table[0, [first + j for j in line]]])
        short.seq_lens[0] = first + len(line)
        chain = oracle.verify_tree(short, q[:, line], [len(line)], [[2 ** (k + 1) - 1 for k in range(len(line))]])
        np.testing.assert_allclose(tree["out"][0, i], chain["out"][0, -1], rtol=1e-12)
        np.testing.assert_allclose(tree["lse"][0, i], chain["lse"][0, -1], rtol=1e-12)


def test_a_node_that_sees_nothing_and_weights_that_sum_to_one():
    w = make("empty", 9, [3], Hq=2, Hkv=1, D=64, q="f32", kv="f32")
    q = np.random.default_rng(0).standard_normal((1, 3, 2, 64))
    r = oracle.verify_tree(w, q, [3], [[0, 2, 7]])
    assert not r["out"][0, 0].any() and np.isneginf(r["lse"][0, 0]).all()
    np.testing.assert_allclose(r["scores"][0, 0].sum(), 2 / 3)          # two of the three nodes have a share


def test_the_codes_of_a_moved_row():
    """The nearest code, ties to even, on all codes and ratios: against torch's cast."""
    from oracle.tree_oracle import _encode
    table = oracle.e4m3_table().astype(np.float32)
    for ratio in (1.0, 0.5, 0.75, 0.33333334, 2.0 ** -9, 0.0):
        x = table[~np.isnan(table)] * np.float32(ratio)
        want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(_encode(x), want), ratio


def test_commit_by_hand():
    """Tokens 0..3 and nodes 4..7; nodes 1 and 3 were accepted."""
    w = make("commit", 2, [8], Hq=1, Hkv=1, D=64, P=4, q="f32", kv="f32")
    rows = lambda pool, t: pool[w.block_table[0, t // 4], 0, t % 4]
    r = oracle.tree_commit(w, [4], np.array([[1, 3, -1, 0]]), [4], scores=np.arange(8, dtype=np.float32).reshape(1, 1, 8))
    assert r["new_lens"][0] == 6 and r["scores"][0, 0].tolist() == [0, 1, 2, 3, 5, 7, 6, 7]
    for t, was in enumerate([0, 1, 2, 3, 5, 7, 6, 7]):
        assert np.array_equal(rows(r["k_pool"], t), rows(w.k_pool, was)) and np.array_equal(rows(r["v_pool"], t), rows(w.v_pool, was))


def test_eviction_by_hand():
    """Six old tokens and two new ones, room for five: position 0 is a sink, the newest is protected; of the others the three heaviest stay."""
    w = make("evict", 2, [8], Hq=1, Hkv=1, D=64, P=4, q="f32", kv="f32")
    weights = np.array([[[0.0, 4.0, 1.0, 2.0, 8.0, 1.0, 77.0, 77.0]]], dtype=np.float32)
    positions = np.array([[[0, 3, 5, 6, 7, 9, -1, -1]]], dtype=np.int32)
    scores = np.array([[[0, 0, 3, 0, 0, 0, 2, 0]]], dtype=np.float32)
    r = oracle.evict_kv(w, scores, 0.5, [6], [5], 1, 1, weights, positions)
    # weights become 0, 2, 3.5, 1, 4, 0.5 | 2, 0; kept: slots 0 (sink), 7 (newest), 4, 2 and 1 (2 as slot 6 has, and the lower slot)
    assert r["new_lens"][0] == 5
    assert r["weights"][0, 0].tolist() == [0.0, 2.0, 3.5, 0.0, 4.0, 1.0, 77.0, 77.0]
    assert r["positions"][0, 0].tolist() == [0, 3, 5, 11, 7, 9, -1, -1]
    rows = lambda pool, t: pool[w.block_table[0, t // 4], 0, t % 4]
    for t, was in enumerate([0, 1, 2, 7, 4]):
        assert np.array_equal(rows(r["k_pool"], t), rows(w.k_pool, was))


def test_an_evicted_fp8_row_keeps_its_value_to_half_a_step():
    w = make("fp8", 4, [60], Hq=1, Hkv=1, D=64, P=16, kv="fp8_e4m3")
    rng = np.random.default_rng(1)
    weights, positions = np.zeros((1, 1, 60), np.float32), np.zeros((1, 1, 60), np.int32)
    scores = rng.random((1, 1, 60), dtype=np.float32)
    r = oracle.evict_kv(w, scores, 1.0, [0], [25], 0, 0, weights, positions)
    table = oracle.e4m3_table()
    for slot in range(25):
        was, at, to = int(r["positions"][0, 0, slot]), w.block_table[0], int(r["positions"][0, 0, slot])
        old = table[w.k_pool[at[was // 16], 0, was % 16]] * w.k_scale[at[was // 16], 0]
        scale = r["k_scale"][at[slot // 16], 0]
        new = table[r["k_pool"][at[slot // 16], 0, slot % 16]] * scale
        assert (np.abs(new - old) <= 2.0 ** -4 * np.abs(old) * (1 + 1e-6) + 2.0 ** -10 * scale).all(), (slot, to)


# ---------------------------------------------------------------- refusals ----
def test_tree_arguments(lib):  # noqa: F811
    s = good_kv()
    def vt(kv=s, q=FAKE, n=8, visible=FAKE, out=FAKE, scores=FAKE, stride=1024, ws=FAKE, wsz=1 << 40):
        return lib.pillar_verify_tree(C.byref(kv), q, n, None, visible, out, None, scores, stride, ws, wsz, None)
    assert vt(q=None) == vt(visible=None) == vt(out=None) == vt(n=0) == vt(stride=1023) == pb.PILLAR_EINVAL
    assert vt(n=65) == pb.PILLAR_EUNSUPPORTED
    assert vt(kv=good_kv(batch=65536)) == pb.PILLAR_EUNSUPPORTED
    assert vt(kv=good_kv(batch=65535, max_seq_len=1 << 20, block_table_stride=1 << 16), stride=1 << 20) == pb.PILLAR_EUNSUPPORTED      # too many units to count
    assert vt(ws=None) == vt(ws=FAKE + 8) == vt(wsz=100) == pb.PILLAR_EWORKSPACE
    for bad in (dict(batch=0), dict(k_pool=None), dict(flags=8), dict(sm_scale=0.0)):
        assert vt(kv=good_kv(**bad)) == pb.PILLAR_EINVAL
    assert lib.pillar_verify_tree(None, FAKE, 8, None, FAKE, FAKE, None, None, 0, FAKE, 1 << 40, None) == pb.PILLAR_EINVAL
    need = lambda kv, n: lib.pillar_tree_workspace_bytes(C.byref(kv), n)
    assert need(s, 8) > 0 and need(s, 8) % 256 == 0 and need(s, 0) == need(s, 65) == need(good_kv(batch=0), 8) == 0
    assert vt(wsz=need(s, 8) - 1) == pb.PILLAR_EWORKSPACE
    assert vt() == vt(out=FAKE + 16) == vt(q=FAKE + 16) == pb.PILLAR_EINVAL                    # queries that would be written over


@pytest.mark.parametrize("kw", [dict(), dict(num_q_heads=128), dict(num_q_heads=8, head_dim=64), dict(q_dtype=pb.PILLAR_F32, kv_dtype=pb.PILLAR_F32)])
def test_a_tree_workspace_does_for_anything_smaller(lib, kw):  # noqa: F811
    need = lambda n, **more: lib.pillar_tree_workspace_bytes(C.byref(good_kv(**{**kw, **more})), n)
    sizes = [need(n) for n in range(1, 65)]
    assert sizes == sorted(sizes)
    for n in (1, 7, 64):
        sizes = [need(n, batch=b) for b in range(1, 200)]
        assert sizes == sorted(sizes)
        sizes = [need(n, max_seq_len=top) for top in range(1, 1025)]
        assert sizes == sorted(sizes)


def test_commit_arguments(lib):  # noqa: F811
    s = good_kv()
    def tc(kv=s, n=8, path=FAKE, lens=FAKE, m=8, now=FAKE * 2, scores=None, stride=0):
        return lib.pillar_tree_commit(C.byref(kv), None, n, path, lens, m, now, scores, stride, None)
    assert tc(path=None) == tc(lens=None) == tc(now=None) == tc(m=0) == tc(n=0) == pb.PILLAR_EINVAL
    assert tc(scores=FAKE, stride=1000) == pb.PILLAR_EINVAL
    assert tc(n=65) == tc(m=65) == pb.PILLAR_EUNSUPPORTED
    assert tc(now=FAKE) == tc(now=FAKE + 12) == tc(now=FAKE - 12) == pb.PILLAR_EINVAL          # the lengths that are being read
    assert tc(kv=good_kv(stride_slot=132)) == tc(kv=good_kv(k_pool=FAKE + 2)) == pb.PILLAR_EUNSUPPORTED


def test_eviction_arguments(lib):  # noqa: F811
    s = good_kv()
    def ev(kv=s, scores=FAKE, stride=1024, decay=0.5, old=FAKE, budgets=FAKE, sink=4, recent=64, weights=FAKE, positions=FAKE, state=1024, now=FAKE,
           ws=FAKE, wsz=1 << 40):
        return lib.pillar_evict_kv(C.byref(kv), scores, stride, decay, old, budgets, sink, recent, weights, positions, state, now, ws, wsz, None)
    assert ev(old=None) == ev(budgets=None) == ev(weights=None) == ev(positions=None) == ev(now=None) == pb.PILLAR_EINVAL
    assert ev(decay=-0.5) == ev(decay=float("nan")) == ev(decay=float("inf")) == ev(sink=-1) == ev(recent=-1) == pb.PILLAR_EINVAL
    assert ev(stride=1023) == ev(state=1023) == pb.PILLAR_EINVAL
    assert ev(kv=good_kv(stride_head=2052)) == ev(kv=good_kv(v_pool=FAKE + 8)) == ev(kv=good_kv(batch=70000)) == pb.PILLAR_EUNSUPPORTED
    assert ev(ws=None) == ev(ws=FAKE + 16) == ev(wsz=64) == pb.PILLAR_EWORKSPACE
    need = lib.pillar_evict_workspace_bytes(C.byref(s))
    assert need > 0 and need % 256 == 0 and ev(wsz=need - 1) == pb.PILLAR_EWORKSPACE
    assert lib.pillar_evict_workspace_bytes(C.byref(good_kv(head_dim=96))) == 0 == lib.pillar_evict_workspace_bytes(None)


def test_the_binding_refuses_what_the_c_side_cannot_see():
    """Types, shapes and strides, before any pointer is passed on."""
    B, Hq, Hkv, D, N, M = 2, 4, 2, 64, 3, 2
    pool = torch.zeros(8, Hkv, 16, D)
    ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    kv = pb.KvCache(k_pool=pool, v_pool=pool, block_table=ints(B, 4), seq_lens=ints(B), num_q_heads=Hq, q_dtype="f32", kv_dtype="f32", sm_scale=0.1,
                    max_seq_len=64)
    ws = torch.empty(1, dtype=torch.uint8)
    q, words, rows = torch.zeros(B, N, Hq, D), torch.zeros(B, N, dtype=torch.int64), torch.zeros(B, Hkv, 64)
    tree = dict(q=q, tree_sizes=ints(B), visible=words, out=q.clone(), lse=torch.zeros(B, N, Hq), scores=rows, workspace=ws)
    for bad in (dict(q=q.double()), dict(q=q.transpose(1, 2)), dict(q=q[:, :2]), dict(visible=words.int()), dict(visible=words[:1]), dict(tree_sizes=ints(B + 1)),
                dict(out=q.to(torch.bfloat16)), dict(lse=torch.zeros(B, Hq, N)), dict(scores=torch.zeros(B, Hkv, 63)), dict(scores=rows.double())):
        with pytest.raises(ValueError):
            pb.pillar_verify_tree(kv, **{**tree, **bad})
    commit = dict(tree_sizes=ints(B), max_nodes=N, path=ints(B, M), path_lens=ints(B), new_lens=ints(B), scores=rows)
    for bad in (dict(path=ints(B, M).long()), dict(path=ints(M, B).t()), dict(path_lens=ints(1)), dict(new_lens=ints(B).float()), dict(scores=torch.zeros(B, 64))):
        with pytest.raises(ValueError):
            pb.pillar_tree_commit(kv, **{**commit, **bad})
    evict = dict(scores=rows, decay=0.5, old_lens=ints(B), budgets=ints(B), sink_tokens=1, recent_tokens=1, weights=rows.clone(), positions=ints(B, Hkv, 64),
                 new_lens=ints(B), workspace=ws)
    for bad in (dict(positions=rows), dict(positions=ints(B, Hkv, 65)), dict(weights=rows[:, :, ::2]), dict(budgets=ints(B + 1)), dict(new_lens=ints(B).long()), dict(old_lens=None, weights=None)):
        with pytest.raises((ValueError, pb.PillarError)):
            pb.pillar_evict_kv(kv, **{**evict, **bad})


def test_words_of_a_tree():
    words = ancestors(np.random.default_rng(0), 64)
    assert all(words[i] >> i & 1 and words[i] < 2 ** (i + 1) for i in range(64))
    assert as_int64([[2 ** 63]])[0, 0] == -2 ** 63
