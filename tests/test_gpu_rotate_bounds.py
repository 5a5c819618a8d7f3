"""Rotary positions and appends at the ends of what they take, on the GPU."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle
import paper_2512_01278_amd as pa
from tests.test_gpu_rotate import Append
from tests.tree_cases import make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("P", [16, 64])                   # (rows kept in registers, and read twice)
@pytest.mark.parametrize("scale", [2.0 ** -149, 2.0 ** -130, 2.0 ** -127, 2.0 ** -110, 2.0 ** -100, 2.0 ** -99, 2.0 ** -98, 0.0])
@pytest.mark.parametrize("fill", [0.0, 1e-30, 2.0 ** -91])
def test_older_tokens_next_to_nothing(P, scale, fill):
    """The page's scale is theirs, their codes stay, and new tokens of nothing are zeros (from 2^-90 / 448 on, what the scale holds)."""
    w = make("tiny", 21, [P + 12, 9], Hq=2, Hkv=2, D=64, P=P, kv="fp8_e4m3", q="f32")
    w.k_scale[:], w.v_scale[:] = scale, scale
    a = Append(w, [4, 3], fused=False)
    a.k[:], a.v[:] = fill, -fill
    a.rows = torch.cat([a.q, a.k, a.v], dim=1).cpu()
    a.run()
    a.check()
    for pool, at, was in ((a.kv.k_pool, a.kv.k_scale, w.k_pool), (a.kv.v_pool, a.kv.v_scale, w.v_pool)):
        for b, first, end in ((0, 8, 12), (1, 6, 9)):
            page = w.block_table[b, 1 if b == 0 else 0]
            assert (at[page] == scale).all() and np.array_equal(pool[page, :, :first].cpu().numpy(), was[page, :, :first])
            new = oracle.e4m3_table()[pool[page, :, first:end].cpu().numpy()]
            assert (np.abs(new * scale) <= 2.0 ** -90).all() and np.isfinite(new).all()
            if scale < 2.0 ** -90 / 448:
                assert (new == 0).all()


TURN = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def unit(position, frequency):
    """Cosine and sine of the very product, reduced in rational numbers."""
    turns = int(position) * Fraction(float(frequency)) / TURN
    angle = float((turns - round(turns)) * TURN)
    return math.cos(angle), math.sin(angle)


@pytest.mark.parametrize("kind", ["one", "model", "large"])
def test_the_farthest_positions(kind):
    """What turns (1, 0) is the cosine and the sine, within 7 * 2^-24 whatever the position: the remainder, at most pi/4, with three roundings on its way into
    fp32 (2.4), the series' last addition and its inner ones (below 3), their ends (2^-29), the amplitude (1)."""
    rng = np.random.default_rng(3)
    f = {"one": 1.0 + rng.uniform(-0.05, 0.05, 32), "model": 1e4 ** (-np.arange(32) / 32), "large": 10.0 ** rng.uniform(0, 9, 32)}[kind]
    f[0] = 1.0
    positions = np.concatenate([2 ** 31 - 1 - rng.integers(0, 1 << 20, 60), -2 ** 31 + rng.integers(0, 1 << 20, 60), rng.integers(-2 ** 31, 2 ** 31, 60), [2 ** 31 - 1, -2 ** 31, 0, 1, -1]])
    x = torch.zeros(len(positions), 1, 64, device=DEV)
    x[..., :32] = 1.0
    out = torch.empty_like(x)
    pa.pillar_rotate(x, torch.tensor(positions, dtype=torch.int32, device=DEV), pa.Rope(torch.from_numpy(f).to(DEV), False, 0.75), out)
    want = 0.75 * np.array([[unit(p, g) for g in f] for p in positions])
    got = out.double().cpu().numpy()[:, 0]
    off = max(np.abs(got[:, :32] - want[..., 0]).max(), np.abs(got[:, 32:] - want[..., 1]).max())
    assert off <= 7 * 2.0 ** -24 * 0.75, f"{off / 0.75 * 2 ** 24:.3g} * 2^-24"
