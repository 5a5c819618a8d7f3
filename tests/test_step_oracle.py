"""New tokens, without a GPU: pins of the oracle, frequencies against their formulas, the rule by which prompts are cut, and refusals."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2512_01278_amd as pa
from oracle import step_oracle as so
from paper_2512_01278_amd import binding as pb
from tests.test_abi import FAKE, good_kv
from tests.test_host_rules import CSRC

INVALID, UNSUPPORTED, WORKSPACE = pb.PILLAR_EINVAL, pb.PILLAR_EUNSUPPORTED, pb.PILLAR_EWORKSPACE
FAR = 1 << 40                  # an address that overlaps with nothing


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pb.LIB_PATH):
        from paper_2512_01278_amd.build import build
        build(verbose=False)
    return pb.load()


# ------------------------------------------------------------- pins ----
def test_a_quarter_turn_by_hand():
    """Frequency pi/2: position 1 turns (a, b) into (-b, a), 2 into (-a, -b), -1 into (b, -a)."""
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    f = np.array([math.pi / 2, 0.0])
    turn = lambda p, il: so.rotate(x, [p], f, interleaved=il)[0, 0]
    assert np.allclose(turn(1, False), [-3, 2, 1, 4, 9]) and np.allclose(turn(2, False), [-1, 2, -3, 4, 9])
    assert np.allclose(turn(1, True), [-2, 1, 3, 4, 9]) and np.allclose(turn(-1, True), [2, -1, 3, 4, 9])
    assert np.allclose(so.rotate(so.rotate(x, [7], f, 2.0), [-7], f, 0.5), x)


def test_logits_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 32))
    f, _ = so.frequencies(32, 1e4)
    at = lambda i, j: float((so.rotate(q, [i], f) * so.rotate(k, [j], f)).sum())
    assert abs(at(5, 2) - at(1005, 1002)) < 1e-9 and abs(at(5, 2) - at(5, 3)) > 1e-3


def test_codes_are_those_of_torchs_cast():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 9, 4000), oracle.e4m3_table()[:127], (oracle.e4m3_table()[:126] + oracle.e4m3_table()[1:127]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(so.encode_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert so.encode_e4m3(np.array([np.nan]))[0] == 127


def test_prompt_rows_are_the_chains():
    """The last k+1 tokens as new ones are the queries of a verification; a whole prompt's last rows are too."""
    w = gen.make_custom(name="chain", seed=3, B=2, Hq=4, Hkv=2, D=64, P=16, spec_k=3, q_dtype="f32", kv_dtype="f32", seq_lens=[37, 4], budgets=[8, 8])
    out, lse, _ = oracle.verify_attn(w)
    q = w.q.astype(np.float64).reshape(8, 4, 64)
    got = so.prompt_attn(w, q, [0, 4, 8])
    assert np.allclose(got["out"].reshape(out.shape), out) and np.allclose(got["lse"].reshape(lse.shape), lse)
    more = np.concatenate([np.random.default_rng(0).standard_normal((33, 4, 64)), q[:4], q[4:]])
    assert np.allclose(so.prompt_attn(w, more, [0, 37, 41])["out"][33:37], out[0])


def test_log_probabilities_by_hand():
    x = np.log(np.array([[1.0, 2.0, 4.0, 1.0]]))
    r = so.logprobs(x, 1.0, np.array([[2, 9, -1]]), 5)
    assert np.allclose(r["lse"], math.log(8)) and np.allclose(r["logprobs"][0, 0], math.log(0.5)) and np.isneginf(r["logprobs"][0, 1:]).all()
    assert np.allclose(r["entropy"], 0.5 * math.log(2) + 0.25 * math.log(4) + 0.25 * math.log(8))
    assert r["top_ids"].tolist() == [[2, 1, 0, 3, -1]]                     # equal ones by number, then nothing
    r = so.logprobs(np.array([[-np.inf, -np.inf], [np.inf, 0.0], [np.nan, 1.0]]), 2.0, np.array([[1], [1], [1]]), 2)
    assert np.isneginf(r["lse"][0]) and r["entropy"][0] == 0 and np.isneginf(r["logprobs"][0]).all() and r["top_ids"][0].tolist() == [0, 1]
    assert r["lse"][1] == np.inf and np.isneginf(r["logprobs"][1, 0]) and np.isnan(r["entropy"][1])
    assert np.isnan(r["lse"][2]) and r["top_ids"][2].tolist() == [1, 0]


# ------------------------------------------------------ frequencies ----
@pytest.mark.parametrize("r", [2, 32, 64, 128, 6])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "ramp", "bands"])
def test_frequencies(lib, r, scaling):
    more = dict(scaling=scaling, factor=4.0, original_len=32768, fast=32.0, slow=1.0)
    f, amplitude = pa.pillar_rope_frequencies(r, 1e6, **more)
    want, factor = so.frequencies(r, 1e6, **more)
    assert f.dtype == torch.float64 and np.allclose(f.numpy(), want, rtol=1e-14, atol=0) and abs(amplitude - factor) < 1e-6


def test_ends_of_the_scalings(lib):
    """The fastest pairs stay, the slowest are stretched by the factor, and what lies between falls."""
    plain, _ = pa.pillar_rope_frequencies(128, 1e4)
    for scaling in ("ramp", "bands"):
        f, a = pa.pillar_rope_frequencies(128, 1e4, scaling, 8.0, 4096, 32.0, 1.0)
        share = (f / plain).numpy()
        assert share[0] == 1.0 and abs(share[-1] - 0.125) < 1e-12 and (np.diff(share) <= 1e-12).all()
        assert abs(a - (0.1 * math.log(8) + 1 if scaling == "ramp" else 1.0)) < 1e-6
    f, _ = pa.pillar_rope_frequencies(128, 1e4, "base", 8.0)
    assert abs(f[-1] / plain[-1] * 8 - 1) < 1e-9 and f[0] == 1.0


def test_frequencies_refuse(lib):
    out, amplitude = (C.c_double * 64)(), C.c_float()
    call = lambda r=128, base=1e4, scaling=0, factor=2.0, n=4096, fast=32.0, slow=1.0, to=out, a=C.byref(amplitude): \
        lib.pillar_rope_frequencies(r, base, scaling, factor, n, fast, slow, to, a)
    assert call() == 0
    for bad in (dict(r=0), dict(r=7), dict(r=-2), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(to=None), dict(a=None),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=math.nan), dict(scaling=3, n=0), dict(scaling=4, slow=0.0),
                dict(scaling=3, fast=1.0), dict(scaling=4, fast=math.inf), dict(scaling=3, base=1.0)):
        assert call(**bad) == INVALID, bad
    assert call(scaling=5) == UNSUPPORTED and call(scaling=-1) == UNSUPPORTED
    with pytest.raises(KeyError):
        pa.pillar_rope_frequencies(64, 1e4, "other")


# ------------------------------------------------------------ the rule ----
MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include "prompt_rules.hpp"
int main(int argc, char** v) {
  const pillar::PromptSteps p(atoi(v[1]), atoi(v[2]), atoi(v[3]), atoi(v[4]), atoi(v[6]));
  printf("%d %d\n", p.tiles, p.units());
  for (int r = 0; r < p.tiles; ++r) printf("%d %d\n", p.steps(r), p.before(r));
  const int units = p.units();
  for (int u = 0; u < units; u += units > 5000 ? 37 : 1) printf("%d %d\n", u, p.tile_of(u));
  printf("%d %d\n", pillar::tile_tokens_shift(256, atoi(v[5])), pillar::tile_tokens_shift(32, atoi(v[5])));
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("prompt_rules")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "rule")], check=True)
    return lambda *args: [tuple(map(int, line.split())) for line in
                          subprocess.run([str(d / "rule"), *map(str, args)], check=True, capture_output=True, text=True).stdout.splitlines()]


@pytest.mark.parametrize("setup", [0, 2])
@pytest.mark.parametrize("q_shift,t_shift", [(0, 6), (1, 7), (4, 6), (5, 6), (6, 6), (7, 6), (8, 6), (3, 7)])
@pytest.mark.parametrize("length,n", [(1, 1), (64, 64), (65, 65), (1000, 1000), (1000, 1), (4097, 513), (130, 129), (5, 9), (200, 1000), (0, 3), (7, 0), (30000, 700)])
def test_units_of_a_prompt(rule, length, n, q_shift, t_shift, setup):
    """Against the definition: every tile's steps reach its last row's token, never past the cache, and each unit has its tile."""
    lines = rule(length, n, q_shift, t_shift, 5, setup)
    Q, T = 1 << q_shift, 1 << t_shift
    tiles = -(-n // Q) if length > 0 else 0
    steps = [s for s, _ in lines[1:1 + tiles]]
    first = length - n
    for r, s in enumerate(steps):
        need = -(-max(0, min(length, first + (r + 1) * Q)) // T)
        assert s >= need and s <= -(-length // T) and (s == need or first < 0), (r, s, need)
    steps = [s + setup for s in steps]
    assert lines[0] == (tiles, sum(steps))
    assert [b for _, b in lines[1:1 + tiles]] == [sum(steps[:r]) for r in range(tiles)]
    ends = np.cumsum(steps)
    for u, tile in lines[1 + tiles:-1]:
        assert tile == int(np.searchsorted(ends, u, side="right"))
    assert lines[-1] == (5, 2)                             # groups of five: 32 tokens of 256 rows, 4 of 32


def test_units_of_a_very_long_context_do_not_overflow(rule):
    lines = rule(16_000_000, 40, 4, 6, 16, 0)
    assert lines[0][0] == 3 and abs(lines[0][1] - 3 * 250_000) <= 3
    assert lines[-1] == (4, 1)


# ------------------------------------------------------------ refusals ----
def rope(**kw):
    r = pb.pillar_rope_t(128, 0, 1.0, 0, FAKE)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_ROPES = [(dict(rotary_dim=0), INVALID), (dict(rotary_dim=127), INVALID), (dict(rotary_dim=130), INVALID), (dict(layout=2), UNSUPPORTED),
             (dict(amplitude=math.inf), INVALID), (dict(amplitude=math.nan), INVALID), (dict(frequencies=None), INVALID),
             (dict(frequencies=FAKE + 4), INVALID), (dict(reserved=1), INVALID)]


def test_rotate_refuses(lib):
    def call(x=FAKE, xs=4096, tokens=10, heads=32, D=128, dtype=pb.PILLAR_BF16, pos=FAKE, r=rope(), out=FAR, os=4096):
        return lib.pillar_rotate(x, xs, tokens, heads, D, dtype, pos, None if r is None else C.byref(r), out, os, None)
    for bad in (dict(x=None), dict(xs=4095), dict(tokens=-1), dict(heads=0), dict(D=0), dict(D=127), dict(pos=None), dict(r=None), dict(out=None), dict(os=4095),
                dict(out=FAKE + 16), dict(out=FAKE, os=8192), dict(out=FAKE - 4096 * 2)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dtype=pb.PILLAR_FP8_E4M3), dict(D=514, xs=32 * 514, os=32 * 514, r=rope()), dict(heads=70000, xs=70000 * 128, os=70000 * 128)):
        assert call(**bad) == UNSUPPORTED, bad
    for bad, code in BAD_ROPES:
        assert call(r=rope(**bad)) == code, bad
    assert call(tokens=0) == pb.PILLAR_OK and call(tokens=0, x=None, out=None, pos=None) == pb.PILLAR_OK


def test_append_refuses(lib):
    def call(kv=None, r=rope(), starts=FAKE, T=20, most=5, pos=None, q=FAKE, qs=4096, qo=FAR, k=2 * FAR, ks=1024, v=3 * FAR, vs=1024):
        return lib.pillar_append_rotated(C.byref(kv or good_kv()), None if r is None else C.byref(r), starts, T, most, pos, q, qs, qo, k, ks, v, vs, None)
    assert lib.pillar_append_rotated(None, None, FAKE, 20, 5, None, None, 0, None, FAKE, 1024, FAKE, 1024, None) == INVALID
    for bad in (dict(T=-1), dict(most=0), dict(starts=None, most=6), dict(k=None), dict(v=None), dict(q=None), dict(qo=None), dict(qs=4095), dict(ks=1023), dict(vs=1023),
                dict(qo=FAKE + 16), dict(qo=FAKE, qs=6144), dict(k=FAR + 64), dict(v=FAR - 64), dict(kv=good_kv(batch=0))):
        assert call(**bad) == INVALID, bad
    for bad in (dict(q=FAKE + 8), dict(qo=FAR + 2), dict(k=2 * FAR + 4), dict(ks=1028), dict(vs=1025), dict(qs=4100), dict(kv=good_kv(stride_slot=130)),
                dict(kv=good_kv(k_pool=FAKE + 8)), dict(kv=good_kv(batch=70000))):
        assert call(**bad) == UNSUPPORTED, bad
    for bad, code in BAD_ROPES:
        assert call(r=rope(**bad)) == code, bad
    assert call(r=rope(rotary_dim=66), kv=good_kv(head_dim=64, stride_slot=128)) == INVALID
    assert call(kv=good_kv(kv_dtype=pb.PILLAR_FP8_E4M3)) == INVALID                        # without scales
    assert call(T=0) == pb.PILLAR_OK and call(T=0, q=None, qo=None, k=None, v=None) == pb.PILLAR_OK


def test_prompt_refuses(lib):
    need = lambda kv=None, T=1000, most=500: lib.pillar_prompt_workspace_bytes(C.byref(kv or good_kv()), T, most)

    def call(kv=None, q=FAKE, starts=FAKE, T=1000, most=500, out=FAR, ws=FAKE, size=1 << 40):
        return lib.pillar_prompt_attn(C.byref(kv or good_kv()), q, starts, T, most, out, None, ws, size, None)
    for bad in (dict(q=None), dict(out=None), dict(T=-1), dict(most=0), dict(starts=None), dict(out=FAKE), dict(out=FAKE + 1024), dict(kv=good_kv(batch=0)), dict(kv=good_kv(flags=8))):
        assert call(**bad) == INVALID, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(size=need() - 1)):
        assert call(**bad) == WORKSPACE, bad
    # more units of work than 32 bits count
    huge = good_kv(batch=60000, num_kv_heads=32, num_q_heads=32, block_table_stride=1 << 20, max_seq_len=1 << 24)
    assert call(kv=huge) == UNSUPPORTED and need(huge) == 0
    assert call(kv=good_kv(batch=70000)) == UNSUPPORTED and call(kv=good_kv(head_dim=96, stride_slot=96)) == UNSUPPORTED
    assert call(T=0) == pb.PILLAR_OK and call(T=0, q=None, out=None) == pb.PILLAR_OK
    assert need(T=-1) == 0 and need(most=0) == 0 and need(good_kv(batch=0)) == 0 and need() > 0


def test_lse_over_the_queries_is_refused(lib):
    q = 4 * FAR                # (room for lse below it: an address does not go below 0)
    for lse in (q, q + 1000 * 32 * 128 * 2 - 4, q - 1000 * 32 * 4 + 4):
        assert lib.pillar_prompt_attn(C.byref(good_kv()), q, FAKE, 1000, 500, FAR, lse, 2 * FAR, 1 << 40, None) == INVALID, lse


def test_workspace_of_a_prompt_does_for_smaller_ones(lib):
    need = lambda T, most, B=4, top=1024: lib.pillar_prompt_workspace_bytes(C.byref(good_kv(batch=B, max_seq_len=top)), T, most)
    for T, most, B, top in ((1, 1, 1, 1), (4, 1, 4, 1024), (100, 30, 4, 700), (1000, 1000, 1, 1000)):
        assert need(T, most, B, top) <= need(1000, 1000)
    need = lambda rows, vocab, top: lib.pillar_logprobs_workspace_bytes(rows, vocab, top)
    sizes = [need(r, 50000, 8) for r in (1, 2, 3, 10, 100, 255, 256, 257, 512, 1000, 5000)]
    assert all(s > 0 for s in sizes)
    for rows in (1, 7, 300, 2000):
        assert need(rows, 50000, 1) <= need(rows, 50000, 8) <= need(rows, 50000, 64)


def test_logprobs_refuse(lib):
    def call(x=FAKE, dtype=pb.PILLAR_BF16, rows=5, vocab=1000, stride=1000, scale=1.0, tok=FAKE, m=2, lp=FAKE, top=4, ids=FAKE, tlp=FAKE, ws=FAKE, size=1 << 30):
        return lib.pillar_token_logprobs(x, dtype, rows, vocab, stride, scale, tok, m, lp, None, None, top, ids, tlp, ws, size, None)
    for bad in (dict(x=None), dict(rows=-1), dict(vocab=0), dict(stride=999), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(tok=None), dict(lp=None),
                dict(m=0), dict(m=-1), dict(top=0), dict(top=-1), dict(ids=None), dict(tlp=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dtype=pb.PILLAR_FP8_E4M3), dict(top=65), dict(x=FAKE + 1), dict(x=FAKE + 2, dtype=pb.PILLAR_F32)):
        assert call(**bad) == UNSUPPORTED, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(size=lib.pillar_logprobs_workspace_bytes(5, 1000, 4) - 1)):
        assert call(**bad) == WORKSPACE, bad
    assert call(rows=0) == pb.PILLAR_OK and call(rows=0, x=None) == pb.PILLAR_OK
    need = lib.pillar_logprobs_workspace_bytes
    assert need(-1, 10, 1) == 0 and need(1, 0, 1) == 0 and need(1, 10, -1) == 0 and need(1, 10, 65) == 0 and need(0, 10, 0) > 0


def test_more_than_a_grid_or_32_bits_hold_is_refused(lib):
    """Work-items of a launch are counted in 32 bits, 256 to a workgroup; numbers of logits and given tokens in 32 bits with a sign, also a step past the end."""
    groups, tokens, room = 1 << 24, (1 << 30) + 1, 1 << 60
    assert lib.pillar_rotate(FAKE, 128, groups, 1, 128, pb.PILLAR_BF16, FAKE, C.byref(rope()), FAKE, 128, None) == UNSUPPORTED
    fp8 = dict(kv_dtype=pb.PILLAR_FP8_E4M3, k_scale=FAKE, v_scale=FAKE)

    def append(kv, rows, q=None):
        return lib.pillar_append_rotated(C.byref(kv), None, FAKE, rows, 1 << 28, None, q, 4096, q and 1 << 50, 1 << 52, 1024, 1 << 54, 1024, None)
    assert append(good_kv(), groups) == UNSUPPORTED and append(good_kv(**fp8), groups, FAKE) == UNSUPPORTED
    assert append(good_kv(max_seq_len=1 << 28, block_table_stride=1 << 24, **fp8), 1 << 28) == UNSUPPORTED         # 2^24 pages and more, without queries
    need = lib.pillar_logprobs_workspace_bytes

    def call(rows=1, vocab=10, m=0):
        return lib.pillar_token_logprobs(FAKE, pb.PILLAR_BF16, rows, vocab, vocab, 1.0, m and FAKE, m, m and 1 << 50, None, None, 0, None, None, FAKE, room, None)
    for bad in (dict(rows=groups), dict(vocab=tokens), dict(m=tokens), dict(rows=2**31 - 1), dict(vocab=2**31 - 1), dict(m=2**31 - 1)):
        assert call(**bad) == UNSUPPORTED, bad
    assert need(groups, 10, 1) == 0 and need(1, tokens, 1) == 0 and need(groups - 1, 10, 1) > 0 and need(1, tokens - 1, 1) > 0


def test_results_over_logits_or_tokens_are_refused(lib):
    rows, vocab, m, top = 3, 1000, 5, 4
    x, tok, apart = FAKE, 2 * FAR, [(3 + i) * FAR for i in range(5)]
    for at in range(5):
        size = 4 * rows * (m, 1, 1, top, top)[at]
        for bad in (x, x + 2 * rows * vocab - 4, x - size + 4, tok, tok + 4 * rows * m - 4, tok - size + 4):
            o = [bad if i == at else apart[i] for i in range(5)]
            assert lib.pillar_token_logprobs(x, pb.PILLAR_BF16, rows, vocab, vocab, 1.0, tok, m, *o[:3], top, *o[3:], 20 * FAR, 1 << 30, None) == INVALID, (at, bad)


def cpu_cache(q="bf16", kv="bf16"):
    pool = torch.zeros(8, 2, 16, 64, dtype={"bf16": torch.bfloat16, "f32": torch.float32}[kv])
    return pa.KvCache(k_pool=pool, v_pool=pool.clone(), block_table=torch.zeros(2, 4, dtype=torch.int32), seq_lens=torch.zeros(2, dtype=torch.int32),
                      num_q_heads=4, q_dtype=q, kv_dtype=kv, sm_scale=0.125, max_seq_len=64)


def test_the_binding_asks_for_types_and_shapes(lib, monkeypatch):
    """On tensors in host memory, as where there is no GPU: each is refused before the library is called."""
    monkeypatch.setattr(torch.cuda, "is_available", lambda: False)
    class Uncalled:
        def __getattr__(self, name):
            return lambda *args: pytest.fail(f"{name} was called")
    monkeypatch.setattr(pb, "load", Uncalled)
    kv, bf, i32 = cpu_cache(), torch.bfloat16, torch.int32
    f = torch.ones(32, dtype=torch.float64)
    x, pos = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, dtype=i32)
    good = pa.Rope(f)
    for args in ((x.half(), pos, good, x.clone()), (x[0], pos, good, x.clone()), (x, pos.long(), good, x.clone()), (x, pos[:5], good, x.clone()), (x, pos, pa.Rope(f.float()), x.clone()),
                 (x, pos, good, x[:, :2]), (x, pos, good, x.float()), (x.transpose(0, 1), pos[:4], good, x.transpose(0, 1)), (x, pos, pa.Rope(f[None]), x.clone())):
        with pytest.raises(ValueError):
            pa.pillar_rotate(*args)
    k = torch.zeros(6, 2, 64, dtype=bf)
    for more in (dict(k_new=k[:5]), dict(v_new=k.float()), dict(k_new=k[:, :1]), dict(starts=torch.zeros(2, dtype=i32)), dict(starts=torch.zeros(3)), dict(positions=pos[:2]), dict(q=x[:, :2]),
                 dict(q=x, q_out=x[:4]), dict(q=x, q_out=x.float()), dict(k_new=k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            pa.pillar_append_rotated(kv, good, **{**dict(k_new=k, v_new=k.clone(), max_new=3), **more})
    ws = torch.zeros(64, dtype=torch.uint8)
    for q, out, lse, starts in ((x.float(), x, None, None), (x[:, :2], x, None, None), (x, x[:3], None, None), (x, x.clone(), torch.zeros(6, 3), None), (x, x.clone(), None, pos[:2])):
        with pytest.raises(ValueError):
            pa.pillar_prompt_attn(kv, q, 3, out, lse, ws, starts=starts)
    z = torch.zeros(3, 100)
    lp, ids = torch.zeros(3, 2), torch.zeros(3, 2, dtype=i32)
    for logits, more in ((z.half(), {}), (z[0], {}), (z.t(), {}), (z, dict(tokens=ids)), (z, dict(tokens=ids.long(), logprobs=lp)), (z, dict(tokens=ids, logprobs=lp[:2])),
                         (z, dict(top_ids=ids)), (z, dict(top_ids=ids, top_logprobs=lp.double())), (z, dict(lse=lp)), (z, dict(entropy=torch.zeros(3, dtype=torch.float64)))):
        with pytest.raises(ValueError):
            pa.pillar_token_logprobs(logits, ws, **more)
