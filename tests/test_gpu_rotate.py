"""Rotary positions and the write of new tokens into the cache, on the GPU, against the oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2512_01278_amd as pa
from oracle import step_oracle as so
from tests.tree_cases import QT, cache_of, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def stored(x, dtype):
    """fp32 values as the type holds them."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(QT[dtype])


def turned_bound(x, positions, f, amplitude, interleaved):
    """How far fp32 arithmetic may be from the rotation of x, element by element.

    The angle's remainder is at most pi/4 and has three roundings on its way into fp32 (2.4 u of the sine or cosine), the series' last addition and its inner
    ones are below 3 u, their ends below 2^-29, the amplitude one u: 7 u of a (|x1| + |x2|); the products and their sum two more.  The angle
    itself has three roundings of 64 bits."""
    m = len(f)
    y = np.abs(x)
    one, two = (np.arange(m) * 2, np.arange(m) * 2 + 1) if interleaved else (np.arange(m), np.arange(m) + m)
    both = (y[..., one] + y[..., two]) * abs(amplitude) * (10 * U + 4 * 2.0 ** -53 * np.abs(np.asarray(positions, dtype=np.float64)[:, None, None] * f))
    bound = np.zeros_like(y)
    bound[..., one], bound[..., two] = both, both
    return bound


def check_rotated(got, want, bound, dtype, what):
    got = got.double().cpu().numpy()
    off = np.abs(got - want) - bound - HALF[dtype] * (np.abs(want) + bound)
    assert not np.isnan(got).any() and off.max() <= 0, f"{what}: {off.max():.3g} more than its bound off"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,r", [(1, 1, 64, 64), (7, 3, 128, 128), (300, 8, 128, 64), (33, 5, 64, 16), (9, 2, 128, 20), (5, 4, 64, 2), (11, 1, 96, 96), (6, 3, 50, 34),
                                     (3, 2, 512, 512), (2, 65, 6, 4), (4100, 2, 64, 64)])
def test_rotate(dtype, interleaved, T, H, D, r):
    rng = np.random.default_rng(T + D + r)
    x = stored(rng.standard_normal((T, H, D)), dtype)
    positions = rng.choice([0, 1, -1, 17, 511, 4096, 32767, 131072, 1000003, -70001, 2 ** 31 - 1], T)
    f, amplitude = so.frequencies(r, 1e4, "ramp", 4.0, 4096, 32.0, 1.0)
    rope = pa.Rope(torch.from_numpy(f).to(DEV), interleaved, amplitude)
    out = torch.full((T, H, D), float("nan"), dtype=QT[dtype], device=DEV)
    at = torch.tensor(positions, dtype=torch.int32, device=DEV)
    xd = x.to(DEV)
    pa.pillar_rotate(xd, at, rope, out)
    x64 = x.double().numpy()
    bound = turned_bound(x64, positions, f, amplitude, interleaved)
    check_rotated(out, so.rotate(x64, positions, f, amplitude, interleaved), bound, dtype, "out")
    assert torch.equal(out[..., r:], xd[..., r:]) and torch.equal(xd.cpu(), x)
    # in place, and from rows of a wider matrix at an odd distance into another one: the same bits
    pa.pillar_rotate(xd, at, rope, xd)
    assert torch.equal(xd, out)
    wide = torch.full((T, H * D + 5), float("nan"), dtype=QT[dtype], device=DEV)
    to = torch.full((T, H * D + 24), float("nan"), dtype=QT[dtype], device=DEV)
    view = lambda m, off: m[:, off:off + H * D].unflatten(1, (H, D))
    view(wide, 3).copy_(x.to(DEV))
    pa.pillar_rotate(view(wide, 3), at, rope, view(to, 8))
    assert torch.equal(view(to, 8), out)
    assert torch.isnan(to[:, :8]).all() and torch.isnan(to[:, 8 + H * D:]).all()


def test_rotation_back_is_its_gradient():
    """The rotation is linear and its transpose is the rotation by the negative position: <R x, y> = <x, R' y>, and back again is where it began."""
    rng = np.random.default_rng(5)
    x, y = (torch.from_numpy(rng.standard_normal((40, 4, 64)).astype(np.float32)).to(DEV) for _ in range(2))
    at = torch.arange(40, dtype=torch.int32, device=DEV) * 999
    f, _ = pa.pillar_rope_frequencies(64, 1e4)
    rope = pa.Rope(f.to(DEV))
    rx, ry, back = (torch.empty_like(x) for _ in range(3))
    pa.pillar_rotate(x, at, rope, rx)
    pa.pillar_rotate(y, -at, rope, ry)
    pa.pillar_rotate(rx, -at, rope, back)
    left, right = (rx.double() * y.double()).sum(dim=2), (x.double() * ry.double()).sum(dim=2)
    size = (x.double().abs() * 2).sum(dim=2) * y.double().abs().amax(dim=2)
    assert ((left - right).abs() <= 22 * U * size).all()
    pairs = (x[..., :32].abs() + x[..., 32:].abs()).double().repeat(1, 1, 2)
    assert ((back.double() - x.double()).abs() <= 33 * U * pairs).all()
    # against differences: R is linear, so a step of any size will do; directions of one element each
    for i in (0, 5, 33, 63):
        step = torch.zeros_like(x)
        step[..., i] = 1.0
        moved = torch.empty_like(x)
        pa.pillar_rotate(x + step, at, rope, moved)
        slope = ((moved - rx).double() * y.double()).sum(dim=2)
        assert ((slope - ry[..., i].double()).abs() <= 48 * U * (1 + size)).all()


class Append:
    """Device tensors of one append, from a host workload whose cache holds the older tokens."""

    def __init__(self, w, new, seed=0, r=None, interleaved=False, positions=None, with_q=True, fused=True, amplitude=1.25):
        rng = np.random.default_rng(seed)
        self.w, self.starts = w, [sum(new[:b]) for b in range(len(new) + 1)]
        T, self.pad = self.starts[-1], 3
        values = rng.standard_normal((T + self.pad, w.Hq + 2 * w.Hkv, w.D)).astype(np.float32) * 2.0 ** rng.integers(-2, 3, (T + self.pad, 1, 1))
        self.rows = stored(values, w.q_dtype)
        self.kv = cache_of(w)
        if fused:
            dev = self.rows.to(DEV)
            self.q, self.k, self.v = dev[:, :w.Hq], dev[:, w.Hq:w.Hq + w.Hkv], dev[:, w.Hq + w.Hkv:]
        else:
            self.q, self.k, self.v = (self.rows[:, s].contiguous().to(DEV) for s in (slice(0, w.Hq), slice(w.Hq, w.Hq + w.Hkv), slice(w.Hq + w.Hkv, None)))
        if not with_q:
            self.q = None
        self.q_out = torch.full((T + self.pad, w.Hq, w.D), float("nan"), dtype=QT[w.q_dtype], device=DEV) if with_q else None
        tokens = [t for _, t in so.token_of_row(w.seq_lens, self.starts)]
        self.at = tokens if positions is None else positions
        self.positions = None if positions is None else torch.tensor(list(positions) + [0] * self.pad, dtype=torch.int32, device=DEV)
        self.f = np.zeros(0)
        self.rope, self.interleaved, self.amplitude = None, interleaved, amplitude
        if r:
            self.f = so.frequencies(r, 1e4)[0]
            self.rope = pa.Rope(torch.from_numpy(self.f).to(DEV), interleaved, amplitude)
        else:
            self.amplitude = 1.0
        self.most = max(max(new), 1)

    def run(self, stream=None):
        starts = torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        pa.pillar_append_rotated(self.kv, self.rope, self.k, self.v, self.most, starts=starts, positions=self.positions, q=self.q, q_out=self.q_out, stream=stream)

    def check(self):
        w, T = self.w, self.starts[-1]
        rows = self.rows.double().numpy()[:T]
        q64, k64, v64 = rows[:, :w.Hq], rows[:, w.Hq:w.Hq + w.Hkv], rows[:, w.Hq + w.Hkv:]
        turn = lambda x: so.rotate(x, self.at, self.f, self.amplitude, self.interleaved) if self.rope else x
        bound = lambda x: turned_bound(x, self.at, self.f, self.amplitude, self.interleaved) if self.rope else np.zeros_like(x)
        if self.q is not None and T:
            check_rotated(self.q_out[:T], turn(q64), bound(q64), w.q_dtype, "q_out")
        if self.q is not None:
            assert torch.isnan(self.q_out[T:]).all()
        if w.kv_dtype != "fp8_e4m3":
            for name, pool, was, x, off in (("k", self.kv.k_pool, w.k_pool, turn(k64), bound(k64)), ("v", self.kv.v_pool, w.v_pool, v64, np.zeros_like(v64))):
                want, slack = oracle.decode_tensor(was, w.kv_dtype), np.zeros(was.shape)
                touched = np.zeros(was.shape, dtype=bool)
                so.append_plain(w, touched, np.ones_like(x, dtype=bool), self.starts)
                so.append_plain(w, want, x, self.starts)
                so.append_plain(w, slack, off, self.starts)
                got = pool.double().cpu().numpy()
                assert np.array_equal(got[~touched], want[~touched], equal_nan=True), f"{name}: rows that are not new"
                err = np.abs(got - want)[touched] - slack[touched] - HALF[w.kv_dtype] * (np.abs(want) + slack)[touched]
                assert not touched.any() or err.max() <= 0, f"{name}: {err.max():.3g} more than its bound off"
            return
        f32 = np.float32
        for name, pool, scale, was, had, x, off in (
                ("k", self.kv.k_pool, self.kv.k_scale, w.k_pool, w.k_scale, turn(k64), bound(k64)),
                ("v", self.kv.v_pool, self.kv.v_scale, w.v_pool, w.v_scale, v64, np.zeros_like(v64))):
            want, now = was.copy(), had.copy()
            so.append_fp8(w, want, now, x.astype(f32), self.starts)
            got, got_scale = pool.cpu().numpy(), scale.cpu().numpy()
            if not off.any():                              # nothing is rounded on the way: the same bits
                assert np.array_equal(got_scale, now, equal_nan=True), f"{name}: scales"
                a, b = oracle.e4m3_table()[got], oracle.e4m3_table()[want]
                assert np.array_equal(a, b, equal_nan=True), f"{name}: codes"
                continue
            touched = np.zeros(was.shape, dtype=bool)
            so.append_plain(w, touched, np.ones_like(x, dtype=bool), self.starts)
            pages = touched.any(axis=(2, 3))
            assert np.array_equal(got_scale[~pages], had[~pages], equal_nan=True) and np.array_equal(got[~pages], was[~pages]), f"{name}: other pages"
            # a scale is off by what the largest value is; a code by half a step of the true value, and what moved that
            most = off.max() / 448
            assert (np.abs(got_scale - now)[pages] <= most + 2 * U * now[pages]).all(), f"{name}: scales"
            value, slack = np.zeros(was.shape), np.zeros(was.shape)
            so.append_plain(w, value, x, self.starts)
            so.append_plain(w, slack, off, self.starts)
            held = oracle.e4m3_table()[got] * got_scale.astype(np.float64)[:, :, None, None]
            s = np.broadcast_to(got_scale.astype(np.float64)[:, :, None, None], was.shape)
            err = (np.abs(held - value) - slack - (2.0 ** -4 + 4 * U) * (np.abs(value) + slack) - 2.0 ** -10 * s)[touched]
            assert err.max() <= 0, f"{name}: codes {err.max():.3g} more than their bound off"
            older = pages[:, :, None, None] & ~touched     # older rows of touched pages, anew or as they were; what no row is stays
            a, b = oracle.e4m3_table()[got[older]] * s[older], oracle.e4m3_table()[want[older]] * np.broadcast_to(now.astype(np.float64)[:, :, None, None], was.shape)[older]
            same = (a == b) | (np.isnan(a) & np.isnan(b))
            # (both are roundings of one value to steps of nearly one size)
            assert (same | (np.abs(a - b) <= 2.0 ** -3 * np.abs(b) + 2.0 ** -9 * s[older])).all(), f"{name}: older rows"


SHAPES = [
    dict(lens=[1], new=[1]), dict(lens=[17, 40, 33], new=[5, 1, 17]), dict(lens=[64, 16, 100], new=[64, 16, 84]), dict(lens=[30, 9, 500, 3], new=[0, 9, 130, 2]),
    dict(lens=[3, 20], new=[7, 4]),                       # more new rows than tokens: the first ones are skipped
    dict(lens=[48, 80], new=[16, 31]),                    # pages that are filled whole, and in part
]


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "fp8_e4m3"), ("f32", "fp8_e4m3")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("r,interleaved", [(None, False), (64, False), (64, True), (24, False), (6, True)])
def test_append(q, kv, shape, r, interleaved):
    w = make("append", 11, shape["lens"], Hq=6, Hkv=2, D=64, q=q, kv=kv)
    a = Append(w, shape["new"], r=r, interleaved=interleaved)
    a.run()
    a.check()


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
@pytest.mark.parametrize("P", [1, 2, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 8), (64, 16, 1), (128, 5, 1)])
def test_pages_and_heads(kv, P, D, Hq, Hkv):
    w = make("pages", 12, [300, 5, 77, 512], Hq=Hq, Hkv=Hkv, D=D, P=P, kv=kv)
    a = Append(w, [290, 1, 40, 0], r=D, positions=list(range(1000, 1000 + 331)))
    a.run()
    a.check()


@pytest.mark.parametrize("kv", ["f32", "bf16", "fp8_e4m3"])
def test_without_starts_without_queries_dense(kv):
    w = make("even", 13, [40, 37, 64], Hq=4, Hkv=4, D=128, kv=kv, q="f32" if kv == "f32" else "bf16")
    a = Append(w, [12, 12, 12], r=128, with_q=False, fused=False)
    a.pad = 0
    pa.pillar_append_rotated(a.kv, a.rope, a.k[:36], a.v[:36], 12)
    a.check()


def test_queries_in_place():
    w = make("in place", 14, [40, 37], Hq=4, Hkv=2, D=64)
    a = Append(w, [6, 9], r=64, fused=False)
    a.run()
    other = Append(w, [6, 9], r=64, fused=False)
    other.q_out = other.q
    other.run()
    assert torch.equal(other.q[:15], a.q_out[:15]) and torch.equal(other.kv.k_pool.nan_to_num(-9), a.kv.k_pool.nan_to_num(-9))


def test_many_requests_of_one_token():
    """More requests than a wavefront has lanes, some without a new token."""
    rng = np.random.default_rng(15)
    new = [int(n) for n in rng.integers(0, 3, 200)]
    w = make("many", 15, [n + int(m) for n, m in zip(new, rng.integers(1, 40, 200))], Hq=2, Hkv=1, D=64)
    a = Append(w, new, r=64)
    a.run()
    a.check()


def test_strided_pools():
    """Slot-major pages: [page][slot][head][D], and rows further apart than they are long."""
    w = make("strided", 16, [50, 33], Hq=4, Hkv=2, D=64)
    plain, strided = Append(w, [20, 9], r=64), Append(w, [20, 9], r=64)
    for name in ("k_pool", "v_pool"):
        p = getattr(strided.kv, name)
        wide = torch.zeros(p.shape[0], p.shape[2], p.shape[1], 80, dtype=p.dtype, device=DEV)
        view = wide[..., :64].transpose(1, 2)
        view.copy_(p)
        setattr(strided.kv, name, view)
    plain.run()
    strided.run()
    for name in ("k_pool", "v_pool"):
        assert torch.equal(getattr(plain.kv, name).nan_to_num(-9), getattr(strided.kv, name).nan_to_num(-9))


def test_values_that_are_not_finite_in_8_bits():
    """NaN stays, infinities become the largest code and say nothing about the scale; zeros and what is next to nothing give scale 0."""
    w = make("nonfinite", 17, [16, 16, 16, 20], Hq=2, Hkv=2, D=64, kv="fp8_e4m3", q="f32")
    a = Append(w, [16, 16, 16, 4], fused=False)
    a.k[3, 0, 5], a.k[4, 0, 6], a.k[5, 0, 7] = float("nan"), float("inf"), -float("inf")
    a.k[16:32] = 0.0
    a.v[16:32] = 1e-30
    a.v[32:48] = float("inf")
    a.k[48:52] *= 1e30                                    # older rows of the page fall to nothing
    a.rows = torch.cat([a.q, a.k, a.v], dim=1).cpu()
    a.run()
    a.check()
    page = w.block_table[0, 0]
    codes = a.kv.k_pool[page, 0].cpu().numpy()
    assert codes[3, 5] & 127 == 127 and codes[4, 6] == 126 and codes[5, 7] == 254
    assert (a.kv.k_scale[w.block_table[1, 0]] == 0).all() and (a.kv.v_scale[w.block_table[1, 0]] == 0).all()


def test_appended_twice_is_the_same():
    """The second append of the same rows finds the page's scale as the first left it."""
    w = make("twice", 18, [37, 21], Hq=2, Hkv=2, D=128, kv="fp8_e4m3")
    a = Append(w, [9, 2], r=128)
    a.run()
    once = [t.clone() for t in (a.kv.k_pool, a.kv.v_pool, a.kv.k_scale, a.kv.v_scale)]
    a.run()
    assert all(torch.equal(x.nan_to_num(-1), y.nan_to_num(-1)) if x.is_floating_point() else torch.equal(x, y)
               for x, y in zip(once, (a.kv.k_pool, a.kv.v_pool, a.kv.k_scale, a.kv.v_scale)))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_captured_and_replayed_with_other_values(kv):
    w = make("graph", 19, [90, 41], Hq=4, Hkv=2, D=64, kv=kv)
    a = Append(w, [20, 3], r=64)
    a.starts_dev = torch.tensor(a.starts, dtype=torch.int32, device=DEV)
    call = lambda: pa.pillar_append_rotated(a.kv, a.rope, a.k, a.v, a.most, starts=a.starts_dev, q=a.q, q_out=a.q_out)
    was = {n: getattr(a.kv, n).clone() for n in ("k_pool", "v_pool", "k_scale", "v_scale") if getattr(a.kv, n) is not None}
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    base = a.q._base if a.q._base is not None else a.q
    for turn in range(3):
        other = Append(w, [20, 3], seed=turn + 50, r=64)
        base.copy_(other.rows.to(DEV))
        for n, t in was.items():
            getattr(a.kv, n).copy_(t)
        g.replay()
        torch.cuda.synchronize()
        a.rows = other.rows
        a.check()


def test_nothing_to_do():
    """No row at all, and requests of which none has a new token."""
    w = make("nothing", 20, [20, 9], Hq=4, Hkv=2, D=64, kv="fp8_e4m3")
    a = Append(w, [0, 0], r=64)
    was = [t.clone() for t in (a.kv.k_pool, a.kv.v_pool, a.kv.k_scale, a.kv.v_scale)]
    a.run()
    pa.pillar_append_rotated(a.kv, a.rope, a.k[:0], a.v[:0], 1, starts=torch.zeros(3, dtype=torch.int32, device=DEV))
    pa.pillar_rotate(a.q_out[:0], torch.zeros(0, dtype=torch.int32, device=DEV), a.rope, a.q_out[:0])
    assert torch.isnan(a.q_out).all()
    assert all(torch.equal(x.nan_to_num(-1), y.nan_to_num(-1)) if x.is_floating_point() else torch.equal(x, y)
               for x, y in zip(was, (a.kv.k_pool, a.kv.v_pool, a.kv.k_scale, a.kv.v_scale)))


@pytest.mark.parametrize("kv", ["bf16", "fp8_e4m3"])
def test_two_appends_at_once(kv):
    """Two caches on two streams, each several times over."""
    calls = [Append(make("at once", s, [300, 41, 90], Hq=4, Hkv=2, D=128, kv=kv), [200, 3, 90], seed=s, r=128) for s in (21, 22)]
    was = [[t.clone() for t in (c.kv.k_pool, c.kv.v_pool, c.kv.k_scale, c.kv.v_scale) if t is not None] for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    starts = [torch.tensor(c.starts, dtype=torch.int32, device=DEV) for c in calls]
    for turn in range(4):
        for c, before in zip(calls, was):
            for t, x in zip([t for t in (c.kv.k_pool, c.kv.v_pool, c.kv.k_scale, c.kv.v_scale) if t is not None], before):
                t.copy_(x)
            c.q_out.fill_(float("nan"))
        torch.cuda.synchronize()
        for c, at, s in zip(calls, starts, streams):
            pa.pillar_append_rotated(c.kv, c.rope, c.k, c.v, c.most, starts=at, q=c.q, q_out=c.q_out, stream=s)
        torch.cuda.synchronize()
        for c in calls:
            c.check()


def test_a_page_of_one_request_among_many_of_another_length():
    """Pages are found by counting those of the requests before: lengths from none to many pages, more requests than lanes."""
    rng = np.random.default_rng(23)
    new = [int(n) for n in np.where(rng.random(130) < 0.3, 0, rng.integers(1, 80, 130))]
    w = make("uneven", 23, [max(1, n + int(m)) for n, m in zip(new, rng.integers(-3, 40, 130))], Hq=2, Hkv=1, D=64, kv="fp8_e4m3")
    a = Append(w, new, r=64)
    a.run()
    a.check()
