"""Rows whose first token is nearly certain: its log probability, and the row's entropy, are as small as what is left for the others, and exact to as many digits.

Both are about R, the others' share relative to the first's.  With u = 2^-24: an exponent d = scale (x - m) is off by 3 u |d| (difference, scale times log2 e,
product), where |d| < 29 for what carries these rows; the exponential by 2 u; additions of positive numbers by u each: eight of a batch, a lane's batches
(at most 6 here, each of which may bring a new largest, 4 u), 6 over lanes, 3 over wavefronts, and as many again over parts with an exponential
each.  Then log1p, a quotient and a product.  Together less than 87 + 2 + 8 + 30 + 9 + 12 + 8 = 156 u, that is 0.93e-5 of the value itself."""
import numpy as np
import pytest
import torch

import paper_2512_01278_amd as pa
from tests.tree_cases import QT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOUND = 1e-5


def certain_rows(R, V, dtype, scale, at, seed):
    """Row r: 1 - p of its first token is about 10^-(1 + r mod 6); where it has a runner-up, that has half of the rest."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, V)) * 0.5
    runner = np.full(R, -1)
    places = [0, 1, -1, 8, -8, 256, -256, 512, -512, 2048, -2048, 4096, -4096, 700, -700]
    for r in range(R):
        rest, offset = 10.0 ** -(1 + r % 6), (0.0, 31.25, -3000.0)[r % 3 if dtype == "f32" else 0]
        place = places[(r // 6) % len(places)]
        x[r] += np.log(rest * (0.5 if place else 1.0) / V) / scale
        x[r, at] = 0.0
        if place:
            runner[r] = at + place
            x[r, at + place] = np.log(0.5 * rest) / scale
        x[r] += offset
    return torch.from_numpy(x.astype(np.float32)).to(QT[dtype]), np.where(runner < 0, at, runner)


def want_of(x, scale, tokens, top):
    """In 64 bits, the first token's own share kept apart from the others'."""
    z = x.double() * float(np.float32(scale))
    best, ids = torch.sort(z, dim=1, descending=True, stable=True)
    d = best - best[:, :1]
    e = d[:, 1:].exp()
    rest = e.sum(dim=1)
    log_s = torch.log1p(rest)
    entropy = log_s - torch.where(e > 0, e * d[:, 1:], 0.0).sum(dim=1) / (1 + rest)
    lp = z - best[:, :1] - log_s[:, None]
    return {"logprobs": lp.gather(1, tokens.long()), "entropy": entropy, "top_ids": ids[:, :top], "top_logprobs": lp.gather(1, ids[:, :top]), "lse": best[:, 0] + log_s}


def check(x, scale, tokens, top):
    R, V = x.shape
    want = want_of(x, scale, tokens, top)
    logits = x.to(DEV)
    got = {"logprobs": torch.full(tokens.shape, 9.0, device=DEV), "entropy": torch.full((R,), 9.0, device=DEV), "lse": torch.full((R,), 9.0, device=DEV)}
    if top:
        got["top_ids"] = torch.full((R, top), -9, dtype=torch.int32, device=DEV)
        got["top_logprobs"] = torch.full((R, top), 9.0, device=DEV)
    ws = torch.full((pa.pillar_logprobs_workspace_bytes(R, V, top),), 255, dtype=torch.uint8, device=DEV)
    pa.pillar_token_logprobs(logits, ws, tokens=tokens.to(DEV), scale=scale, **got)
    for name in ("logprobs", "entropy") + (("top_logprobs",) if top else ()):
        off = (got[name].double().cpu() - want[name]).abs() / want[name].abs()
        assert off.max() < BOUND, f"{name}: {off.max():.3g} of itself off, row {int(off.reshape(R, -1).amax(dim=1).argmax())}"
    if top:
        assert torch.equal(got["top_ids"].cpu().long(), want["top_ids"])
    assert ((got["lse"].double().cpu() - want["lse"]).abs() < BOUND * want["lse"].abs().clamp(min=1.0)).all()


def tokens_of(R, V, at, runner, seed):
    t = np.random.default_rng(seed + 1).integers(0, V, (R, 3))
    t[:, 0], t[:, 1] = at, runner
    return torch.from_numpy(t.astype(np.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("R,V,at", [(520, 9000, 4500), (4, 50000, 25000), (90, 12000, 6000)])
@pytest.mark.parametrize("scale", [1.0, 1.25])
def test_nearly_certain(dtype, top, R, V, at, scale):
    """A row of one part (520 rows fill the chip) and rows of many; the runner-up beside the first, before and after, in the same 16 bytes, in the same lane's
    next load (256 or 512 away) or next batch (2048 or 4096), and in other lanes."""
    turns = 1 if R >= 90 else 23                           # few rows at a time: all places in turn
    x, runner = certain_rows(R * turns, V, dtype, scale, at, V + top)
    for i in range(turns):
        rows = slice(i * R, (i + 1) * R)
        check(x[rows], scale, tokens_of(R, V, at, runner[rows], i), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_certain_at_the_ends(dtype):
    """The first token among those that are read apart from the row's 16-byte vectors, and rows of a few logits."""
    V = 9001
    for at in (0, 1, V - 1, V - 2):
        x, _ = certain_rows(6, V, dtype, 1.0, 4500, at)
        x[:, [at, 4500]] = x[:, [4500, at]]
        check(x, 1.0, tokens_of(6, V, at, np.full(6, 4500), at), 2)
    for V in (2, 3, 9, 70):
        x = torch.full((6, V), -30.0, dtype=QT[dtype])
        x[:, V // 2] = 0.0
        for r in range(6):
            x[r, V - 1 if V // 2 != V - 1 else 0] = np.log(10.0 ** -(r + 1))
        check(x, 1.0, tokens_of(6, V, V // 2, np.full(6, 0), V), 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_first_tokens(dtype):
    """One of two equal largest logits is the rest of the other."""
    V = 9000
    x = torch.full((5, V), -40.0, dtype=QT[dtype])
    x[:, 4500] = 7.0
    for r, other in enumerate((4501, 4499, 4500 + 512, 4500 - 4096, 100)):
        x[r, other] = 7.0
    check(x, 1.0, tokens_of(5, V, 4500, np.full(5, 100), 3), 2)


def test_rising_and_falling():
    """Every batch brings a new largest, or none does; the last steps are large."""
    V = 9000
    up = torch.linspace(-60.0, -20.0, V)
    x = torch.stack([up, up.flip(0), up, up.flip(0)])
    x[2, -1], x[3, 0] = 0.0, 0.0
    check(x, 1.0, tokens_of(4, V, V - 1, np.zeros(4, dtype=int), 5), 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 9000, 50000])
def test_logits_further_apart_than_their_type_reaches(dtype, V):
    """x - m is beyond the largest number while scale * (x - m) is not."""
    x = torch.full((3, V), -3.0e38, dtype=QT[dtype])
    x[:, V // 2], x[:, 3] = 3.0e38, 0.0
    x[1, 5:20] = 2.5e38
    x[2, ::2] = -1.0e38
    scale = 4.0e-38 if V < 100 else 6.0e-38
    check(x, scale, tokens_of(3, V, V // 2, np.array([3, 7, 4]), V), 3)


def test_a_workspace_for_many_rows_does_for_fewer():
    """One of the largest call's size, with nothing written behind it."""
    V, top = 50000, 8
    size = pa.pillar_logprobs_workspace_bytes(640, V, top)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
    for dtype in (torch.float32, torch.bfloat16):
        x = (torch.randn(640, V, generator=torch.Generator().manual_seed(5)) * 3).to(dtype).to(DEV)
        whole = torch.empty(640, top, device=DEV)
        pa.pillar_token_logprobs(x, ws[:size], top_ids=torch.empty(640, top, dtype=torch.int32, device=DEV), top_logprobs=whole)
        for R in (511, 300, 255, 171, 64, 3, 1):
            ids, lp, lse = torch.empty(R, top, dtype=torch.int32, device=DEV), torch.empty(R, top, device=DEV), torch.empty(R, device=DEV)
            pa.pillar_token_logprobs(x[:R], ws[:size], lse=lse, top_ids=ids, top_logprobs=lp)
            # (other parts, other sums: 2^-24 for each of some 60 additions and of an exponent below 40)
            assert ((lp - whole[:R]).abs() <= 200 * 2.0 ** -24 * whole[:R].abs().clamp(min=1.0)).all(), R
            assert torch.equal(ids[:, 0].long(), x[:R].float().argmax(dim=1)), R
    assert (ws[size:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V", [(520, 9000), (3, 50000)])
def test_a_first_token_that_is_not_far_ahead(dtype, R, V):
    """Up to p = 4/5 a runner-up that comes earlier may stay the reference: the first token is then one of the others' sum, 1 + R up to 5, and log p, 0.22 and more, the
    difference of its logarithm and of 1.39.  A flat rest moves the reference three times at the most: 8 + 6 + 12 + 9 additions and moves and an exponent's 6 u, of which
    R / (1 + R) counts, over 0.22, and 14 u for the difference: 163 u, 0.98e-5."""
    x = torch.full((R, V), float(np.log(0.01 / V)))
    at = V // 2
    runner = np.empty(R, dtype=int)
    for r in range(R):
        p = (0.51, 0.6, 0.7, 0.78, 0.8, 0.82, 0.9)[r % 7]
        runner[r] = at + (-2048, -4096, -512, -1, 1, 512, 2048, 100, -100)[(r // 7) % 9]
        x[r, at], x[r, runner[r]] = float(np.log(p)), float(np.log(0.99 - p))
    check((x + 3.0).to(QT[dtype]), 1.0, tokens_of(R, V, at, runner, R), 2)
