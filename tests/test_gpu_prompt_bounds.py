"""Attention of new tokens at the ends of what it takes, on the GPU."""
import pytest
import torch

from tests.test_gpu_prompt import PromptRun, check_prompt
from tests.tree_cases import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("bf16", "fp8_e4m3"), ("f32", "f32")])
def test_far_more_rows_than_tokens(q, kv):
    """Thousands of tiles whose rows see nothing ahead of the ones that see a few tokens: those are the result of the same rows alone."""
    w = make("beyond", 31, [64, 300], Hq=2, Hkv=1, D=64, q=q, kv=kv)
    few = PromptRun(w, [64, 40], pad=0)
    few.run()
    check_prompt(few)
    many = PromptRun(w, [30000, 40], pad=0)
    many.q[30000 - 64:] = few.q
    many.run()
    first = 30000 - 64
    assert (many.out[:first] == 0).all() and torch.isneginf(many.lse[:first]).all()
    # (another cut into ranges: the same sums in another order, and probabilities rounded against other maxima)
    r = PromptRun(w, [64, 40], pad=0)
    r.out, r.lse = many.out[first:], many.lse[first:]
    check_prompt(r)
