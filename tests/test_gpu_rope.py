"""Norms and rotations of queries and keys (spork_qk_rope) against the definition
in float64: layouts, parts of a head, far positions, strides, in place, rows at no
position, one of queries and keys alone, streams and graphs."""
import numpy as np
import pytest
import torch

from gpu_cases import say
from paper_2607_03333_amd import spork
from rows_cases import to_f64, turn_bound, turned

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SPORK = {BF16: spork.SPORK_DTYPE_BF16, F32: spork.SPORK_DTYPE_F32}
EPS = 1e-6


class Case:
    def __init__(self, dtype, hq, hkv, d, n, rotary, interleaved=False, norm=True, positions=None, magnitude=1.0, base=1e6, seed=0,
                 gap=0, gain=1.5):
        rng = np.random.default_rng(seed * 31 + hq * d + n + rotary)
        normal = lambda *m: torch.from_numpy(rng.standard_normal(m).astype(np.float32))  # noqa: E731
        self.dtype, self.hq, self.hkv, self.d, self.n, self.interleaved = dtype, hq, hkv, d, n, interleaved
        self.shape = spork.make_shape(hq, hkv, d, 16, SPORK[dtype], 1.0)
        self.rows = (normal(n, (hq + 2 * hkv) * d + gap) * gain).to(dtype).cuda()
        self.q = self.rows[:, :hq * d].unflatten(1, (hq, d))
        self.k = self.rows[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        self.pos = np.asarray(rng.integers(0, 131072, n) if positions is None else positions, np.int32)
        self.positions = torch.from_numpy(self.pos).cuda()
        self.inv_freq = spork.spork_rope_frequencies(rotary, base)[0] if rotary else None
        self.magnitude = magnitude
        layout = spork.SPORK_ROPE_INTERLEAVED if interleaved else spork.SPORK_ROPE_HALF
        self.rope = spork.make_rope(torch.from_numpy(self.inv_freq).cuda(), layout, magnitude) if rotary else None
        self.weights = [(1 + 0.3 * normal(d)).to(dtype).cuda() for _ in range(2)] if norm else [None, None]
        self.norm = spork.make_qk_norm(*self.weights, EPS) if norm else None
        self.q_out = torch.full((n, hq, d), 7.5, dtype=dtype, device="cuda")
        self.k_out = torch.full((n, hkv, d), 7.5, dtype=dtype, device="cuda")

    def run(self):
        spork.spork_qk_rope(self.shape, self.rope, self.norm, self.positions, self.q, self.k, self.q_out, self.k_out)

    def reference(self):
        out = []
        for x, w in ((self.q, self.weights[0]), (self.k, self.weights[1])):
            want, size = turned(to_f64(x), None if w is None else to_f64(w), EPS, self.pos, self.inv_freq, self.magnitude,
                                self.interleaved)
            out.append((want, turn_bound(want, size, self.d, self.dtype == BF16)))
        return out

    def check(self, tag, ref=None, outs=None):
        torch.cuda.synchronize()
        rows = self.pos >= 0
        worst = 0.0
        for got, (want, tol) in zip(outs or (self.q_out, self.k_out), ref or self.reference()):
            off = np.abs(to_f64(got) - want) / tol
            assert (off[rows] <= 1).all(), f"{tag}: off by {off[rows].max():.2f} of the bound"
            worst = max(worst, off[rows].max() if rows.any() else 0.0)
            assert (got[torch.from_numpy(~rows).cuda()] == 7.5).all(), f"{tag}: rows at no position"
        say(f"  rope {tag}: at {worst:.2f} of the bound")


HEADS = [(BF16, 32, 8, 128), (BF16, 5, 1, 64), (F32, 4, 2, 64), (F32, 7, 7, 128), (BF16, 16, 16, 64), (BF16, 1, 1, 128)]


@pytest.mark.parametrize("norm", (False, True))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("dtype,hq,hkv,d", HEADS)
def test_every_part_of_a_head(dtype, hq, hkv, d, interleaved, norm):
    for rotary in range(16, d + 1, 16):
        c = Case(dtype, hq, hkv, d, 7, rotary, interleaved, norm, positions=[0, 1, 5, 100, 4097, 131071, -1])
        c.run()
        c.check(f"{rotary} of {d}")


@pytest.mark.parametrize("n", (1, 2, 3, 63, 64, 65, 500, 2049))
@pytest.mark.parametrize("dtype,hq,hkv,d", HEADS[:4])
def test_numbers_of_rows(dtype, hq, hkv, d, n):
    c = Case(dtype, hq, hkv, d, n, d, gap=8)
    c.run()
    c.check(f"{n} rows")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_norms_alone(dtype):
    c = Case(dtype, 6, 2, 128, 9, 0, positions=range(9))
    spork.spork_qk_rope(c.shape, None, c.norm, None, c.q, c.k, c.q_out, c.k_out)
    c.check("norms alone")


def test_positions_at_the_end_of_32_bits():
    """Angles of 2^31 radians: 64 bits hold them to 2^-22 at worst, the magnitude of the rows times that is the bound's
    share for the angle."""
    c = Case(F32, 4, 2, 128, 4, 128, norm=False, positions=[2 ** 31 - 1, 2 ** 30 + 1, 16777217, 1])
    c.run()
    ref = [(w, t + 2.0 ** -21 * np.abs(w).max()) for w, t in c.reference()]
    c.check("far", ref)


@pytest.mark.parametrize("magnitude", (1.1386294361119891, -0.5, 0.0))
def test_magnitudes(magnitude):
    c = Case(BF16, 8, 2, 64, 20, 32, magnitude=magnitude)
    c.run()
    c.check(f"magnitude {magnitude}")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("interleaved", (False, True))
def test_in_place(dtype, interleaved):
    c = Case(dtype, 8, 2, 64, 300, 48, interleaved)
    c.pos[5] = c.pos[77] = -1
    c.positions.copy_(torch.from_numpy(c.pos))
    ref, before = c.reference(), c.rows.clone()
    spork.spork_qk_rope(c.shape, c.rope, c.norm, c.positions, c.q, c.k, c.q, c.k)
    torch.cuda.synchronize()
    assert torch.equal(c.rows[[5, 77]], before[[5, 77]]) and torch.equal(c.rows[:, 10 * 64:], before[:, 10 * 64:])
    c.rows[[5, 77]] = 7.5
    c.check("in place", ref, (c.q, c.k))


def test_queries_or_keys_alone():
    c = Case(BF16, 8, 2, 128, 33, 128)
    norm = spork.make_qk_norm(c.weights[0], None, EPS)
    spork.spork_qk_rope(c.shape, c.rope, norm, c.positions, c.q, None, c.q_out, None)
    torch.cuda.synchronize()
    assert (c.k_out == 7.5).all()
    norm = spork.make_qk_norm(None, c.weights[1], EPS)
    spork.spork_qk_rope(c.shape, c.rope, norm, c.positions, None, c.k, None, c.k_out)
    c.check("alone")


def test_outputs_side_by_side_in_wider_rows():
    c = Case(BF16, 8, 2, 64, 50, 64)
    wide = torch.full((50, 12 * 64), 7.5, dtype=BF16, device="cuda")
    q, k = wide[:, 64:9 * 64].unflatten(1, (8, 64)), wide[:, 9 * 64:11 * 64].unflatten(1, (2, 64))
    spork.spork_qk_rope(c.shape, c.rope, c.norm, c.positions, c.q, c.k, q, k)
    c.check("side by side", outs=(q, k))
    assert (wide[:, :64] == 7.5).all() and (wide[:, 11 * 64:] == 7.5).all()


@pytest.mark.parametrize("eps", (0.0, 1e-50, 1e-6))
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_norms_of_very_small_and_very_large_heads(dtype, d, eps):
    """Squares that 32 bits don't hold, beside heads whose squares they do, and heads that hold both. (Factor and products in
    64 bits: well inside the bound of 32.)"""
    tops = [1e-44 if dtype == F32 else 1e-39, 1e-38, 1e-30, 3e-20, 1e-13, 2e-12, 1.0, 1e12, 5e17, 1e19, 1e30, 2e38]
    c = Case(dtype, 4, 2, d, len(tops), d, gain=0.3)
    for i, top in enumerate(tops):
        c.rows[i, :2 * d] = (c.rows[i, :2 * d].double().clamp(-1, 1) * top).to(dtype)
        c.rows[i, 4 * d:5 * d] = (c.rows[i, 4 * d:5 * d].double().clamp(-1, 1) * top).to(dtype)
        c.rows[i, 2 * d + 5] = top
    # (a head of zeros has no norm without eps)
    for x, w in zip((c.q, c.k), c.weights):
        assert (x.double().abs().amax(-1) > 0).all() and w is not None
    norm = spork.make_qk_norm(*c.weights, eps)
    ref = []
    for x, w in ((c.q, c.weights[0]), (c.k, c.weights[1])):
        want, size = turned(to_f64(x), to_f64(w), eps, c.pos, c.inv_freq, 1.0, False)
        ref.append((want, turn_bound(want, size, d, dtype == BF16)))
    spork.spork_qk_rope(c.shape, c.rope, norm, c.positions, c.q, c.k, c.q_out, c.k_out)
    c.check(f"eps {eps}", ref)


def test_zero_rows_infinities_and_nan():
    """A row of zeros has a norm by eps alone; a head that holds an infinity or a NaN spoils itself and no other."""
    c = Case(BF16, 4, 2, 128, 3, 128)
    c.rows[0, :128] = 0
    ref = c.reference()
    c.rows[1, 128:256][17] = float("inf")
    c.rows[2, 256:384][99] = float("nan")
    c.run()
    torch.cuda.synchronize()
    assert (c.q_out[0, 0] == 0).all()
    assert not torch.isfinite(c.q_out[1, 1]).all() and torch.isnan(c.q_out[2, 2]).all()
    c.q_out[1, 1] = torch.from_numpy(ref[0][0][1, 1])
    c.q_out[2, 2] = torch.from_numpy(ref[0][0][2, 2])
    c.check("spoiled heads", ref)


def test_no_rows():
    c = Case(BF16, 4, 2, 64, 2, 64)
    spork.spork_qk_rope(c.shape, c.rope, c.norm, c.positions[:0], c.q[:0], c.k[:0], c.q_out[:0], c.k_out[:0])
    torch.cuda.synchronize()
    assert (c.q_out == 7.5).all()


def test_streams_and_replays():
    """Two batches in flight on two streams; a graph whose rows and positions change between replays."""
    cases = [Case(BF16, 8, 2, 128, 700, 128, seed=1), Case(F32, 4, 4, 64, 900, 32, True, seed=2)]
    torch.cuda.synchronize()
    for c in cases:
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            c.run()
    for c in cases:
        c.check("two streams")
    c = cases[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for seed in (3, 4, 5):
        other = Case(BF16, 8, 2, 128, 700, 128, seed=seed)
        c.rows.copy_(other.rows)
        c.positions.copy_(other.positions)
        for x, y in zip(c.weights, other.weights):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert torch.equal(c.q_out, other.q_out) and torch.equal(c.k_out, other.k_out)
        other.check(f"replay {seed}")


def test_rows_past_4_gib():
    """Rows that begin beyond 2^32 bytes; those in front of them are at no position."""
    c = Case(BF16, 64, 8, 128, 5, 128)
    n = (1 << 31) // (80 * 128) + 900
    wide = torch.empty(n, 80 * 128, dtype=BF16, device="cuda")
    wide[-5:] = c.rows
    wide[:3] = 7.5
    positions = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    positions[-5:] = c.positions
    q, k = wide[:, :64 * 128].unflatten(1, (64, 128)), wide[:, 64 * 128:72 * 128].unflatten(1, (8, 128))
    ref = c.reference()
    spork.spork_qk_rope(c.shape, c.rope, c.norm, positions, q, k, q, k)
    torch.cuda.synchronize()
    assert (wide[:3] == 7.5).all()
    c.check("past 4 GiB", ref, (q[-5:], k[-5:]))
