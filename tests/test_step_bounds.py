"""What the calls around new tokens ask for and refuse, on the CPU."""
import ctypes as C
import shutil
import subprocess

import pytest

from paper_2512_01278_amd import binding as pb
from tests.test_abi import good_kv
from tests.test_host_rules import CSRC


@pytest.fixture(scope="module")
def lib():
    return pb.load()


def test_a_workspace_of_log_probabilities_does_for_smaller_calls(lib):
    """No call asks for more than one with as many rows, logits and alternatives, or more."""
    need = lib.pillar_logprobs_workspace_bytes
    rows = [1, 2, 3, 10, 85, 100, 128, 170, 171, 255, 256, 257, 300, 511, 512, 513, 640, 5000, 1 << 20]
    vocabs = [1, 100, 2047, 2048, 2052, 4096, 4104, 32000, 50001, 150000, 1 << 20, 1 << 30]
    for top in (0, 1, 8, 64):
        for vocab in vocabs:
            sizes = [need(r, vocab, top) for r in rows]
            assert all(s > 0 for s in sizes) and sizes == sorted(sizes), (vocab, top)
        for r in rows:
            sizes = [need(r, vocab, top) for vocab in vocabs]
            assert sizes == sorted(sizes), (r, top)
    assert need((1 << 24) - 1, 1 << 30, 64) < 1 << 20                  # rows of one part leave nothing there


MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include "prompt_rules.hpp"
// the tile of a unit by halving
static int search(const pillar::PromptSteps& p, int u) {
  int lo = 0, hi = p.tiles;
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (p.before(mid) <= u) lo = mid;
    else hi = mid;
  }
  return lo;
}
int main(int, char** v) {
  const pillar::PromptSteps p(atoi(v[1]), atoi(v[2]), atoi(v[3]), atoi(v[4]), atoi(v[5]));
  const int units = p.units();
  int furthest = 0;
  for (int i = 0; i <= 4000; ++i) {
    const int u = i < 1000 ? i : i < 2000 ? units - 1 - (i - 1000) : (int)((long long)(units - 1) * (i - 2000) / 2000);
    if (u < 0 || u >= units) continue;
    const int off = abs(p.tile_near(u) - search(p, u));
    if (off > furthest) furthest = off;
  }
  printf("%d %d %d\n", p.tiles, units, furthest);
}
"""


@pytest.fixture(scope="module")
def near(tmp_path_factory):
    d = tmp_path_factory.mktemp("tile_near")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run([shutil.which("g++") or "c++", "-O1", "-std=c++17", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "near")], check=True)
    return lambda *args: tuple(map(int, subprocess.run([str(d / "near"), *map(str, args)], check=True, capture_output=True, text=True).stdout.split()))


@pytest.mark.parametrize("q_shift,t_shift,setup", [(0, 7, 1), (1, 7, 1), (3, 7, 1), (0, 6, 1), (4, 6, 4), (5, 6, 4), (6, 6, 4), (7, 6, 4), (8, 6, 4), (6, 6, 0)])
@pytest.mark.parametrize("length,n", [(64, 1 << 20), (1, 1 << 20), (5000, 1 << 20), (1 << 20, 1 << 20), (1 << 20, 70000), (1 << 24, 1000), (300, 299), (100, 5000), (8192, 8192), (40000, 65536)])
def test_a_units_tile_is_found_in_a_few_steps(near, length, n, q_shift, t_shift, setup):
    """However many tiles there are, among them far more rows than tokens in the cache.  Where steps are stairs of T / Q tiles, the sum of what they are off their mean
    is at most a quarter of a stair's width by half its height, T / 8 Q units, and a tile has a step at the least; the root and its rounding are off by two."""
    if -(-n // (1 << q_shift)) * (-(-length // (1 << t_shift)) + setup) >= 1 << 30:
        pytest.skip("more units than a call may have")
    tiles, units, furthest = near(length, n, q_shift, t_shift, setup)
    assert tiles == -(-n // (1 << q_shift)) and 0 < units < 1 << 30
    assert furthest <= 2 + (1 << max(t_shift - q_shift, 0)) // 8, (tiles, units, furthest)


# ------------------------------------------------------------ results over what is read ----
FAR = [i << 40 for i in range(1, 20)]                      # addresses that overlap with nothing


def around(at, bytes_, size, step=4):
    """Addresses, in multiples of `step`, of a result of `size` bytes that lies over what is there, at its first and its last bytes."""
    return at, at + (bytes_ - 1) // step * step, at - size + step


def test_rotated_rows_over_positions_or_frequencies_are_refused(lib):
    tokens, heads, D = 1000, 4, 128
    size = 2 * tokens * heads * D
    x, positions, frequencies = FAR[:3]
    call = lambda out, stride=heads * D, x=x: lib.pillar_rotate(x, heads * D, tokens, heads, D, pb.PILLAR_BF16, positions,
                                                               C.byref(pb.pillar_rope_t(D, 0, 1.0, 0, frequencies)), out, stride, None)
    for at, bytes_ in ((positions, 4 * tokens), (frequencies, 4 * D)):
        for out in around(at, bytes_, size):
            assert call(out) == pb.PILLAR_EINVAL, (at, out)
            assert call(out, x=out) == pb.PILLAR_EINVAL, (at, out)         # (in place too)


def far_kv(**kw):
    """A cache whose arrays lie far apart."""
    more = dict(k_pool=FAR[10], v_pool=FAR[11], block_table=FAR[12], seq_lens=FAR[13])
    if kw.get("kv_dtype") == pb.PILLAR_FP8_E4M3:
        more.update(k_scale=FAR[14], v_scale=FAR[15])
    return good_kv(**more, **kw)


def described(kv):
    """Arrays of the cache that every workgroup reads, and their bytes."""
    spans = [(kv.seq_lens, 4 * kv.batch), (kv.block_table, 4 * ((kv.batch - 1) * kv.block_table_stride + kv.max_seq_len // kv.page_size))]
    return spans + [(at, 4 * kv.num_pages * kv.num_kv_heads) for at in (kv.k_scale, kv.v_scale) if at]


@pytest.mark.parametrize("kv_dtype", [pb.PILLAR_BF16, pb.PILLAR_FP8_E4M3])
def test_rotated_queries_over_what_an_append_reads_are_refused(lib, kv_dtype):
    kv, T = far_kv(kv_dtype=kv_dtype), 400
    size = 2 * T * 32 * 128
    starts, positions, frequencies, q, k, v = FAR[:6]

    def call(q_out, rope=True, positions=positions):
        r = C.byref(pb.pillar_rope_t(128, 0, 1.0, 0, frequencies)) if rope else None
        return lib.pillar_append_rotated(C.byref(kv), r, starts, T, 100, positions, q, 4096, q_out, k, 1024, v, 1024, None)
    for at, bytes_ in [(starts, 4 * 5), (positions, 4 * T), (frequencies, 4 * 128)] + described(kv):
        for out in around(at, bytes_, size, 16):
            assert call(out) == pb.PILLAR_EINVAL, (at, out)


@pytest.mark.parametrize("kv_dtype", [pb.PILLAR_BF16, pb.PILLAR_FP8_E4M3])
def test_attention_of_new_tokens_over_what_it_reads_is_refused(lib, kv_dtype):
    kv, T = far_kv(kv_dtype=kv_dtype), 400
    size = {"out": 2 * T * 32 * 128, "lse": 4 * T * 32}
    q, starts, free, other, ws = FAR[:5]
    call = lambda out, lse: lib.pillar_prompt_attn(C.byref(kv), q, starts, T, 100, out, lse, ws, 1 << 39, None)
    for at, bytes_ in [(q, size["out"]), (starts, 4 * 5)] + described(kv):
        for out in around(at, bytes_, size["out"]):
            assert call(out, None) == pb.PILLAR_EINVAL and call(out, other) == pb.PILLAR_EINVAL, (at, out)
        for lse in around(at, bytes_, size["lse"]):
            assert call(free, lse) == pb.PILLAR_EINVAL, (at, lse)
    for lse in around(free, size["out"], size["lse"]):
        assert call(free, lse) == pb.PILLAR_EINVAL, lse


def test_log_probabilities_over_each_other_are_refused(lib):
    rows, vocab, m, top = 3, 1000, 5, 4
    size = [4 * rows * n for n in (m, 1, 1, top, top)]
    x, tok, ws = FAR[:3]
    for i in range(5):
        for j in range(5):
            for bad in around(FAR[5 + j], size[j], size[i]) if i != j else ():
                o = [bad if k == i else FAR[5 + k] for k in range(5)]
                assert lib.pillar_token_logprobs(x, pb.PILLAR_BF16, rows, vocab, vocab, 1.0, tok, m, *o[:3], top, *o[3:], ws, 1 << 30, None) == pb.PILLAR_EINVAL, (i, j, bad)
