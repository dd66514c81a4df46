"""Writes into the cache of 8-bit codes (spork_kvq_write, spork_kvq_copy_batch)
against the definition in float64, code by code: runs of every length at every
place of a block, scales that grow and stay, codes that are written anew, ties,
infinities, rows behind the last token, strides, streams and graphs.

Codes and scales have to be equal to the model's. Keys that come ready, and
values, are divided by powers of two: exact. Normed and rotated keys are float64 on
both sides, which differ by less than 2^-44 of the row's size: a value so near to
the middle of two codes does not occur here (its chance is below 2^-40 each), and
the model says so if it does."""
import numpy as np
import pytest
import torch

from gpu_cases import say
from paper_2607_03333_amd import spork
from rows_cases import LARGEST, VALUES, PoolModel, _MIDDLE, same_codes, to_f64, turn_bound, turned

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SPORK = {BF16: spork.SPORK_DTYPE_BF16, F32: spork.SPORK_DTYPE_F32}
EPS = 1e-6


class Cache:
    """Pools of random codes and scales on the GPU, and their model."""

    def __init__(self, rng, hkv, d, bs, blocks, low=100, high=130):
        self.hkv, self.d, self.bs, self.blocks = hkv, d, bs, blocks
        kc, vc = (rng.integers(0, 256, (blocks, hkv, bs, d)).astype(np.uint8) for _ in range(2))
        for c in (kc, vc):
            c[c & 127 == 127] = 3  # a number
        ks, vs = (rng.integers(low, high, (blocks, hkv)).astype(np.uint8) for _ in range(2))
        self.k, self.v = PoolModel(kc, ks), PoolModel(vc, vs)
        gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.tensors = dict(k_codes=gpu(kc), v_codes=gpu(vc.swapaxes(2, 3)), k_scale=gpu(ks), v_scale=gpu(vs))
        self.kvq = spork.make_kvq(**self.tensors)

    def check(self, tag):
        torch.cuda.synchronize()
        got = {n: t.cpu().numpy() for n, t in self.tensors.items()}
        assert np.array_equal(got["k_scale"], self.k.scale), f"{tag}: scales of keys"
        assert np.array_equal(got["v_scale"], self.v.scale), f"{tag}: scales of values"
        assert same_codes(got["k_codes"], self.k.codes), f"{tag}: codes of keys"
        assert same_codes(got["v_codes"].swapaxes(2, 3), self.v.codes), f"{tag}: codes of values"


class Step:
    """Runs (block, kept, tokens) of new rows, with queries if there is a rotation or a norm."""

    def __init__(self, dtype, hq, cache, runs, rotary=None, norm=True, interleaved=False, seed=0, gap=0, gains=(0.01, 10.0), behind=0):
        rng = np.random.default_rng(seed + 17 * len(runs) + cache.d)
        hkv, d, bs = cache.hkv, cache.d, cache.bs
        rotary = d if rotary is None else rotary
        self.dtype, self.hq, self.cache, self.runs, self.interleaved = dtype, hq, cache, runs, interleaved
        self.n = sum(r[2] for r in runs)
        rows = self.n + behind
        self.shape = spork.make_shape(hq, hkv, d, bs, SPORK[dtype], 1.0)
        gain = np.exp(rng.uniform(*np.log(gains), (rows, 1)))
        x = rng.standard_normal((rows, (hq + 2 * hkv) * d + gap)) * gain
        self.rows = torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()
        part = lambda a, h: self.rows[:, a * d:(a + h) * d].unflatten(1, (h, d))  # noqa: E731
        self.q, self.k_new, self.v_new = part(0, hq), part(hq, hkv), part(hq + hkv, hkv)
        slots = [b * bs + kept + i for b, kept, m in runs for i in range(m)] + [-1] * behind
        self.pos = np.concatenate([rng.integers(0, 100000, self.n), np.full(behind, -1)]).astype(np.int32)
        self.slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
        self.positions = torch.from_numpy(self.pos).cuda()
        self.inv_freq = spork.spork_rope_frequencies(rotary, 1e6)[0] if rotary else None
        layout = spork.SPORK_ROPE_INTERLEAVED if interleaved else spork.SPORK_ROPE_HALF
        self.rope = spork.make_rope(torch.from_numpy(self.inv_freq).cuda(), layout, 1.125) if rotary else None
        weight = lambda: torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(dtype).cuda()  # noqa: E731
        self.weights = (weight(), weight()) if norm else (None, None)
        self.norm = spork.make_qk_norm(*self.weights, EPS) if norm else None
        self.turns = bool(rotary or norm)
        self.q_out = torch.full((rows, hq, d), 7.5, dtype=dtype, device="cuda")
        self.bad = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self):
        spork.spork_kvq_write(self.shape, self.cache.kvq, self.rope, self.norm, self.slots, self.positions if self.rope else None,
                              self.q if self.turns else None, self.k_new, self.v_new, self.q_out if self.turns else None, self.bad)

    def turned(self, x, which):
        w = self.weights[which]
        return turned(to_f64(x[:self.n]), None if w is None else to_f64(w), EPS, self.pos[:self.n], self.inv_freq, 1.125, self.interleaved)

    def model(self):
        k, v, row = self.turned(self.k_new, 1)[0], to_f64(self.v_new[:self.n]), 0
        for block, kept, m in self.runs:
            self.cache.k.write(block, kept, k[row:row + m])
            self.cache.v.write(block, kept, v[row:row + m])
            if self.turns:  # no key lies so near to a middle that 64 bits could differ
                x = np.abs(k[row:row + m]) * 2.0 ** -self.cache.k.e[block].astype(np.float64)[:, None]
                if not self.norm:
                    x = x[..., :2 * len(self.inv_freq)]  # the others are as they came
                at = np.searchsorted(_MIDDLE, x)
                near = [np.abs(_MIDDLE[np.clip(at - i, 0, 125)] - x) < 2.0 ** -40 * x for i in (0, 1)]
                assert not np.count_nonzero(near)
            row += m

    def check(self, tag):
        self.cache.check(tag)
        assert self.bad.item() == len(self.slots) - self.n
        if not self.turns:
            assert (self.q_out == 7.5).all()
            return
        want, size = self.turned(self.q, 0)
        off = np.abs(to_f64(self.q_out[:self.n]) - want) / turn_bound(want, size, self.cache.d, self.dtype == BF16)
        assert (off <= 1).all(), f"{tag}: queries off by {off.max():.2f} of the bound"
        assert (self.q_out[self.n:] == 7.5).all(), f"{tag}: rows behind the last"
        say(f"  kvq write {tag}: queries at {off.max():.2f} of the bound")


def do(dtype, hq, hkv, d, bs, runs, tag, blocks=None, **kw):
    rng = np.random.default_rng(kw.get("seed", 0) + hkv * d + bs)
    c = Cache(rng, hkv, d, bs, blocks or max(r[0] for r in runs) + 3)
    s = Step(dtype, hq, c, runs, **kw)
    s.run()
    s.model()
    s.check(tag)
    return s


SHAPES = [(BF16, 8, 2, 128, 16), (BF16, 5, 5, 64, 32), (F32, 4, 2, 64, 16), (F32, 3, 1, 128, 32), (BF16, 7, 1, 128, 32), (BF16, 4, 4, 64, 16)]


@pytest.mark.parametrize("ready", (False, True))
@pytest.mark.parametrize("dtype,hq,hkv,d,bs", SHAPES)
def test_every_place_of_a_block(dtype, hq, hkv, d, bs, ready):
    """A run from every place to every other: each in a block of its own."""
    places = [(kept, m) for kept in range(bs) for m in range(1, bs - kept + 1)]
    runs = [(3 * i % len(places) if len(places) % 3 else i, kept, m) for i, (kept, m) in enumerate(places)]
    do(dtype, hq, hkv, d, bs, runs, "places", rotary=0 if ready else None, norm=not ready, blocks=len(places) + 1)


@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("dtype,hq,hkv,d,bs", SHAPES[:4])
def test_parts_of_a_head(dtype, hq, hkv, d, bs, interleaved):
    for rotary, norm in [(r, n) for r in range(0, d + 1, 16) for n in (False, True) if r or n]:
        do(dtype, hq, hkv, d, bs, [(1, 3, 9), (2, 0, bs), (4, bs - 1, 1)], f"{rotary} of {d}", rotary=rotary, norm=norm,
           interleaved=interleaved, seed=rotary)


@pytest.mark.parametrize("dtype,hq,hkv,d,bs", SHAPES)
def test_prompts_and_single_tokens(dtype, hq, hkv, d, bs):
    """Sequences of one token to many blocks in one step, rows behind the last one, projections with a gap."""
    rng = np.random.default_rng(d + bs)
    free, runs = iter(rng.permutation(400)), []
    for new, held in [(1, 0), (1, 5), (3 * bs + 5, 0), (1, bs - 1), (2 * bs, 7), (1, bs), (bs, 0), (9 * bs + 1, 2), (2, bs - 1), (1, 1)]:
        at = held
        while at < held + new:
            m = min(held + new, (at // bs + 1) * bs) - at
            runs.append((int(next(free)), at % bs, m))
            at += m
    for seed, gap, behind in ((0, 0, 0), (1, 16, 40)):
        do(dtype, hq, hkv, d, bs, runs, "prompts", blocks=400, seed=seed, gap=gap, behind=behind)


@pytest.mark.parametrize("rows", (600, 3000))
@pytest.mark.parametrize("dtype,hq,hkv,d,bs", SHAPES[:3])
def test_many_rows(dtype, hq, hkv, d, bs, rows):
    """Launches whose workgroups take several rows: one sequence, and a token in each of many blocks."""
    runs, at = [], 5
    while at < rows:
        m = min(rows, (at // bs + 1) * bs) - at
        runs.append((at // bs, at % bs, m))
        at += m
    do(dtype, hq, hkv, d, bs, runs, "one long prompt")
    do(dtype, hq, hkv, d, bs, [(i, i % bs, 1) for i in range(rows)], "single tokens")


@pytest.mark.parametrize("rows", (768, 769, 1600, 6200, 12300))
@pytest.mark.parametrize("dtype,hq,hkv,d,bs", [(BF16, 2, 1, 64, 16), (F32, 1, 1, 64, 32), (BF16, 9, 9, 64, 16)])
def test_windows_of_every_width(dtype, hq, hkv, d, bs, rows):
    """Runs of all lengths one behind the other, in launches whose workgroups take one to sixteen rows."""
    rng = np.random.default_rng(rows)
    runs, n = [], 0
    while n < rows:
        kept = int(rng.choice((0, 0, 1, bs - 1, rng.integers(0, bs))))
        m = min(int(rng.choice((1, 2, bs, bs))), bs - kept, rows - n)
        runs.append((len(runs), kept, m))
        n += m
    do(dtype, hq, hkv, d, bs, runs, f"{rows} rows", behind=3)


@pytest.mark.parametrize("dtype,hq,hkv,d,bs", SHAPES)
def test_token_by_token(dtype, hq, hkv, d, bs):
    """A block filled one token at a time, scales growing at some of them, and then begun again."""
    rng = np.random.default_rng(bs + d)
    c = Cache(rng, hkv, d, bs, 3)
    for i in range(2 * bs + 3):
        s = Step(dtype, hq, c, [(1, i % bs, 1)], rotary=0, norm=False, seed=i, gains=(0.001, 1000.0))
        s.run()
        s.model()
        s.check(f"token {i}")


def test_scales_at_their_borders():
    """Largest magnitudes at, just below and just above 448 times a power of two, zeros, the smallest and largest numbers."""
    tops = [448.0, 447.9999, 448.0001, 1.75, 1.7500001, 1.0, 0.0, 1e-45, 2.0 ** -126, 2.0 ** -110, 2.0 ** -92, 3.4e38, 2.0 ** 127, 2.0 ** 120]
    rng = np.random.default_rng(3)
    for bs, kept in ((16, 0), (16, 4), (32, 31)):
        c = Cache(rng, 1, 64, bs, len(tops), low=27, high=40)
        s = Step(F32, 2, c, [(i, kept, 1) for i in range(len(tops))], rotary=0, norm=False)
        for i, t in enumerate(tops):
            x = rng.uniform(-1, 1, (2, 64)).astype(np.float32)
            x[0, 5], x[1, 63] = 1, -1
            s.k_new[i, 0], s.v_new[i, 0] = (torch.from_numpy(np.float32(t) * y).cuda() for y in x)
        s.run()
        s.model()
        s.check("borders")


def test_every_middle_of_two_codes():
    """Ties go to the even code, and values one place off a middle to the code on their side."""
    middles = np.concatenate([_MIDDLE, -_MIDDLE]).astype(np.float32)
    around = np.concatenate([middles, np.nextafter(middles, np.float32(np.inf)), np.nextafter(middles, np.float32(-np.inf)),
                             VALUES[:127].astype(np.float32)])
    x = np.zeros((len(around) // 63 + 1, 64), np.float32)
    x[:, 0] = LARGEST  # the scale is 1
    x[:, 1:].reshape(-1)[:len(around)] = around
    rng = np.random.default_rng(4)
    c = Cache(rng, 1, 64, 16, len(x))
    s = Step(F32, 1, c, [(i, 0, 1) for i in range(len(x))], rotary=0, norm=False)
    s.k_new[:, 0] = s.v_new[:, 0] = torch.from_numpy(x).cuda()
    s.run()
    s.model()
    s.check("middles")


@pytest.mark.parametrize("grows", (1, 2, 5, 9, 30, 200))
def test_codes_written_anew(grows):
    """Every code in front of a token that raises the scale by 2^grows."""
    rng = np.random.default_rng(grows)
    c = Cache(rng, 2, 128, 32, 2, low=27, high=28)
    for pool, name in ((c.k, "k_codes"), (c.v, "v_codes")):
        every = np.arange(256).astype(np.uint8)
        pool.codes[1, :, :30] = np.resize(every, (2, 30, 128))
        c.tensors[name][1] = torch.from_numpy(np.ascontiguousarray(pool.codes[1] if name == "k_codes" else pool.codes[1].swapaxes(1, 2)))
    s = Step(F32, 4, c, [(1, 30, 1)], rotary=0, norm=False)
    top = np.float32(LARGEST * 2.0 ** (27 - 127 + grows))
    for x in (s.k_new, s.v_new):
        x.copy_(torch.clamp(x, -1, 1) * float(top))
        x[:, :, 9] = float(top)
    s.run()
    s.model()
    s.check(f"anew 2^{grows}")


@pytest.mark.parametrize("dtype", (BF16, F32))
def test_infinities_and_nan(dtype):
    """They become codes that are no number, count nothing for the scale, and change no other code."""
    c = Cache(np.random.default_rng(5), 2, 64, 16, 4)
    s = Step(dtype, 4, c, [(0, 0, 16), (1, 3, 2), (2, 15, 1)], rotary=0, norm=False)
    for x, at in ((s.k_new, 3), (s.v_new, 8)):
        x[at, 0, 5], x[at, 1, 63], x[at + 9, 0, 1] = float("nan"), float("inf"), float("-inf")
    s.k_new[18] = float("nan")
    s.run()
    s.model()
    s.check("infinities")


def test_slots_outside_the_pool():
    c = Cache(np.random.default_rng(6), 2, 64, 16, 4)
    s = Step(BF16, 4, c, [(0, 0, 5), (2, 6, 3)], behind=4)
    slots = s.slots.clone()
    s.slots[8:] = torch.tensor([4 * 16, -1, 1 << 40, -(1 << 62)], device="cuda")
    s.positions[8:] = 7
    s.run()
    s.model()
    s.check("slots outside")
    s.slots.copy_(slots)


def test_slots_that_name_a_block_twice_stay_in_bounds():
    """Rows that give a block's tokens in no order, and a slot twice: what that block holds is undefined, no other changes."""
    c = Cache(np.random.default_rng(7), 2, 64, 16, 5)
    s = Step(BF16, 4, c, [(0, 0, 5), (2, 0, 16), (3, 1, 2)])
    s.slots[5:21] = 2 * 16 + torch.tensor([3, 3, 2, 1, 0, 15, 14, 3, 4, 5, 5, 6, 0, 0, 9, 8], device="cuda")
    s.run()
    s.model()
    torch.cuda.synchronize()
    for name, pool in (("k_codes", c.k), ("v_codes", c.v)):
        got = c.tensors[name][2].cpu().numpy()
        pool.codes[2] = got if name == "k_codes" else got.swapaxes(1, 2)
    c.k.e[2], c.v.e[2] = (c.tensors[n][2].cpu().numpy().astype(np.int64) - 127 for n in ("k_scale", "v_scale"))
    s.check("twice")


def test_queries_in_place_and_left_out():
    c = Cache(np.random.default_rng(8), 2, 128, 16, 6)
    s = Step(BF16, 8, c, [(0, 0, 16), (1, 2, 7), (4, 0, 1)], gap=24)
    want = s.turned(s.q, 0)
    s.model()
    keep = s.rows.clone()
    spork.spork_kvq_write(s.shape, c.kvq, s.rope, spork.make_qk_norm(None, s.weights[1], EPS), s.slots, s.positions, None, s.k_new, s.v_new,
                          None)
    c.check("without queries")
    assert torch.equal(s.rows, keep)
    spork.spork_kvq_write(s.shape, c.kvq, s.rope, s.norm, s.slots, s.positions, s.q, s.k_new, s.v_new, s.q)
    c.check("the same again")
    off = np.abs(to_f64(s.q) - want[0]) / turn_bound(*want, 128, True)
    assert (off <= 1).all() and torch.equal(s.rows[:, 8 * 128:], keep[:, 8 * 128:])


def test_no_rows():
    c = Cache(np.random.default_rng(9), 1, 64, 16, 2)
    s = Step(BF16, 2, c, [(0, 0, 2)])
    spork.spork_kvq_write(s.shape, c.kvq, s.rope, s.norm, s.slots[:0], s.positions[:0], s.q[:0], s.k_new[:0], s.v_new[:0], s.q_out[:0])
    c.check("no rows")


@pytest.mark.parametrize("hkv,d,bs", [(2, 128, 16), (3, 64, 32), (1, 64, 16), (2, 128, 32)])
def test_copies(hkv, d, bs):
    """Every number of tokens; entries that are no copies are skipped, and so are those behind *n_copies."""
    c = Cache(np.random.default_rng(hkv + d + bs), hkv, d, bs, 2 * bs + 4)
    copies = [(bs + i, i, i + 1) for i in range(bs)]
    wrong = [(0, 0, 3), (-1, 1, 3), (1, 2 * bs + 4, 3), (2, 3, 0), (2, 3, bs + 1), (1 << 30, 4, 1)]
    for src, dst, n in copies:
        c.k.copy(src, dst, n)
        c.v.copy(src, dst, n)
    listed = torch.tensor(copies + wrong + [(5, 2 * bs + 1, 4)], dtype=torch.int32, device="cuda")
    n = torch.tensor([len(listed) - 1], dtype=torch.int32, device="cuda")
    spork.spork_kvq_copy_batch(spork.make_shape(hkv, hkv, d, bs, spork.SPORK_DTYPE_BF16, 1.0), c.kvq, listed, n)
    c.check("copies")


def test_streams_and_replays():
    """Two caches written on two streams at once; one graph whose rows, slots and positions change between replays."""
    steps = []
    for i, (dtype, hq, hkv, d, bs) in enumerate(SHAPES[:2]):
        c = Cache(np.random.default_rng(i), hkv, d, bs, 80)
        steps.append(Step(dtype, hq, c, [(j, j % bs, min(3, bs - j % bs)) for j in range(70)], seed=i))
    torch.cuda.synchronize()
    for s in steps:
        with torch.cuda.stream(torch.cuda.Stream()):
            s.run()
    for s in steps:
        s.model()
        s.check("two streams")
    s = steps[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for i in range(4):
        other = Step(BF16, 8, s.cache, [(j, (j + i) % 16, min(3, 16 - (j + i) % 16)) for j in range(30)], seed=20 + i)
        other.n = sum(r[2] for r in other.runs)
        s.slots.fill_(-1)
        s.bad.zero_()
        for name in ("rows", "slots", "positions"):
            getattr(s, name)[:other.n].copy_(getattr(other, name))
        for x, y in zip(s.weights, other.weights):
            x.copy_(y)
        s.q_out.fill_(7.5)
        s.n, s.runs = other.n, other.runs
        s.pos = s.positions.cpu().numpy()
        torch.cuda.synchronize()
        graph.replay()
        s.model()
        s.check(f"replay {i}")


def test_blocks_past_4_gib():
    """Blocks whose codes begin beyond 2^32 bytes, and a copy between them."""
    hkv, d, bs, used = 8, 128, 32, 5
    c = Cache(np.random.default_rng(11), hkv, d, bs, used)
    nb = (1 << 32) // (hkv * d * bs) + 1000
    big = {n: torch.zeros((nb, *t.shape[1:]), dtype=torch.uint8, device="cuda") for n, t in c.tensors.items()}
    for n, t in c.tensors.items():
        big[n][-used:] = t
    kvq = spork.make_kvq(**big)
    s = Step(BF16, 8, c, [(0, 0, 32), (1, 5, 4), (3, 31, 1)])
    slots = s.slots + (nb - used) * bs
    spork.spork_kvq_write(s.shape, kvq, s.rope, s.norm, slots, s.positions, s.q, s.k_new, s.v_new, s.q_out)
    copies = torch.tensor([[nb - 2, nb - 3, 9]], dtype=torch.int32, device="cuda")
    spork.spork_kvq_copy_batch(s.shape, kvq, copies, torch.ones(1, dtype=torch.int32, device="cuda"))
    for n, t in c.tensors.items():
        t.copy_(big[n][-used:])
    s.model()
    c.k.copy(3, 2, 9)
    c.v.copy(3, 2, 9)
    s.check("past 4 GiB")
    assert not any(t[:-used].any() for t in big.values())
