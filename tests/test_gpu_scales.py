"""fp8 pages whose scale is zero, or far from the others', on the GPU: trees, commit and eviction."""
import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2512_01278_amd as pa
from tests.test_gpu_evict import State
from tests.test_gpu_tree import committed
from tests.tree_cases import TreeRun, ancestors, check_tree, make

pytestmark = pytest.mark.gpu

GENERIC = pa.PILLAR_FLAG_GENERIC_KERNELS
SMALLEST = 2.0 ** -80                  # a v_scale below counts as that


def verified(run, what):
    print(f"[case] {what}", flush=True)
    run.run()
    torch.cuda.synchronize()
    return check_tree(run, what)


def heaviest_page(w, run, b):
    """Index of the page that holds the token of the largest probability of request b."""
    p = oracle.verify_tree(w, run.q64, run.sizes, run.words)["scores"][b].max(axis=0)
    return int(np.nanargmax(p)) // w.P


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("N", [1, 9, 40])
@pytest.mark.parametrize("which", ["heaviest", "all", "tree", "context"])
def test_pages_of_zeros(which, N, flags):
    """A page of zeros has codes and scale 0: its tokens keep their weight in lse and scores."""
    lens = [N + 5, 300, 1100]
    w = make("zeros", 41, lens, Hq=4, Hkv=2, D=64, kv="fp8_e4m3")
    words = [ancestors(np.random.default_rng(b), N) for b in range(3)]
    top = [heaviest_page(w, TreeRun(w, N, None, words, seed=N), b) for b in range(3)]
    for b, n in enumerate(lens):
        pages = -(-n // w.P)
        for p in {"heaviest": [top[b]], "all": range(pages), "tree": [pages - 1], "context": range(pages - 1)}[which]:
            w.v_pool[w.block_table[b, p]], w.v_scale[w.block_table[b, p]] = 0, 0.0
    verified(TreeRun(w, N, None, words, seed=N, flags=flags), f"zeros {which} {N}")


def test_a_scale_of_zero_counts_as_the_smallest():
    """Whatever the codes, at most 448 times the smallest scale of each token's weight; and nothing of it in fp32 arithmetic."""
    for flags in (0, GENERIC):
        w = make("zero", 42, [70, 500], Hq=4, Hkv=1, D=64, kv="fp8_e4m3")
        w.v_scale[w.block_table[w.block_table >= 0]] = 0.0
        run = TreeRun(w, 5, None, [ancestors(np.random.default_rng(b), 5) for b in range(2)], flags=flags)
        run.run()
        torch.cuda.synchronize()
        assert run.out.abs().max() <= (0.0 if flags else 448 * SMALLEST * (1 + 2.0 ** -6))
        want = oracle.verify_tree(w, run.q64, run.sizes, run.words)
        assert np.abs(run.lse.double().cpu().numpy() - want["lse"]).max() <= (64 * want["reach"] + 600 + 8 * np.abs(want["lse"]).max()) * 2.0 ** -24


@pytest.mark.parametrize("flags", [0, GENERIC])
@pytest.mark.parametrize("N", [1, 9, 40])
def test_light_tokens_of_a_page_of_zeros_beside_a_heavy_one_of_a_large_scale(N, flags):
    """2000 tokens, each 2^-20 of the first one's weight: two thousandths of the sum, which the log-sum-exp and the scores have to have."""
    w = make("wide", 43, [2000], Hq=1, Hkv=1, D=64, kv="fp8_e4m3", q="bf16")
    w.k_pool[:], w.k_scale[:] = 0, 1.0
    w.v_pool[w.block_table[0]], w.v_scale[w.block_table[0]] = 0, 0.0
    w.k_pool[w.block_table[0, 0], 0, 0, :] = 0x38                              # 1.0
    w.v_scale[w.block_table[0, 0]] = 4096.0
    w.v_pool[w.block_table[0, 0], 0, :16] = 0x3c                               # 1.5
    q = np.full((1, N, 1, 64), 20 * np.log(2) / (64 * w.sm_scale), dtype=np.float32)
    bits = gen.bf16_bits_from_f32(q)
    run = TreeRun(w, N, None, [[2 ** (i + 1) - 1 for i in range(N)]], flags=flags,
                  queries_of=(torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16), gen.f32_from_bf16_bits(bits).astype(np.float64)))
    verified(run, f"wide {N}")


def zero_some(w, share, seed):
    rng = np.random.default_rng(seed)
    for name in ("k_scale", "v_scale"):
        scale = getattr(w, name)
        scale[rng.random(scale.shape) < share] = 0.0
    return w


@pytest.mark.parametrize("P", [1, 4, 16])
def test_commit_between_pages_of_zeros(P):
    rng = np.random.default_rng(P)
    lens, sizes = [64, 65, 300, 131, 40], [40, 30, 50, 3, 40]
    for share in (0.5, 1.0):
        w = zero_some(make("commit0", P, lens, kv="fp8_e4m3", D=64, P=P, Hq=4, Hkv=2), share, P)
        path = np.stack([rng.integers(0, s, size=12) for s in sizes])
        committed(w, 64, sizes, path, [12, 7, 12, 2, 0], with_scores=False)


@pytest.mark.parametrize("P", [1, 16, 64])
def test_eviction_between_pages_of_zeros(P):
    for share in (0.5, 1.0):
        w = zero_some(make("evict0", P, [40, 41, 300, 77, 256], kv="fp8_e4m3", D=64, P=P, Hq=4, Hkv=2), share, P)
        State(w, P).check([30, 41, 290, 0, 255], [30, 20, 200, 64, 100], 2, 4, what=f"zeros P={P} {share}")
