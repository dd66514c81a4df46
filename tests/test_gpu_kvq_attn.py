"""Attention of the new tokens of a ragged batch over the cache of 8-bit codes
(spork_kvq_attn) against the definition in float64, over the values that the codes
and scales stand for: the cases of the attention over the other pools, scales from
block to block far apart, every code, and the same values in bf16 pools.

Codes become bf16 or float32 exactly, so the bounds are those of the other pools'
attention (paged_cases.bounds)."""
import math

import numpy as np
import pytest
import torch

import test_gpu_chunk
from gpu_cases import say
from paged_cases import attention, blocks_of, bounds
from paper_2607_03333_amd import spork
from rows_cases import VALUES, encode
from test_gpu_chunk import BF16, EDGES, F32, SPORK

pytestmark = pytest.mark.gpu


def coded_pools(rng, hkv, d, bs, kv, spare=3, junk=127, scales=(119, 123)):
    """Codes and scales of every sequence's context in shuffled blocks, `junk` codes wherever no token lies; the table, and
    the contexts as float64 [tokens][hkv][d] pairs. Blocks of no sequence have scales that are no number."""
    held = [blocks_of(k, bs) for k in kv]
    nb = sum(held) + spare
    order = rng.permutation(nb)
    table = np.full((len(kv), max(held + [1])), -7, np.int32)
    codes = [np.full((nb, hkv, bs, d), junk, np.uint8) for _ in range(2)]
    scale = [np.full((nb, hkv), 255, np.uint8) for _ in range(2)]
    contexts, at = [], 0
    for s, (length, h) in enumerate(zip(kv, held)):
        ids = order[at:at + h]
        at += h
        table[s, :h] = ids
        parts = []
        for c, e in zip(codes, scale):
            x = encode(np.clip(rng.standard_normal((h, hkv, bs, d)) * 100, -448, 448))
            e[ids] = rng.integers(*scales, (h, hkv))
            for j, b in enumerate(ids):
                m = min(bs, length - j * bs)
                c[b, :, :m] = x[j, :, :m]
            values = VALUES[x] * 2.0 ** (e[ids].astype(np.float64) - 127)[:, :, None, None]
            parts.append(torch.from_numpy(values.swapaxes(1, 2).reshape(h * bs, hkv, d)[:length].copy()))
        contexts.append(tuple(parts))
    gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    pools = dict(k_codes=gpu(codes[0]), v_codes=gpu(codes[1].swapaxes(2, 3)), k_scale=gpu(scale[0]), v_scale=gpu(scale[1]))
    return pools, gpu(table), contexts


class Case(test_gpu_chunk.Case):
    def __init__(self, dtype, hq, hkv, d, bs, new, kv, seed=0, gain=1.0, scale=None, spare_rows=3, gap=0, junk=127, scales=(119, 123)):
        rng = np.random.default_rng(seed * 977 + hq + d + bs + sum(kv) % 1009)
        self.dtype, self.new, self.kv = dtype, list(new), list(kv)
        self.scale = float(np.float32(1.0 / math.sqrt(d) if scale is None else scale))
        self.shape = spork.make_shape(hq, hkv, d, bs, SPORK[dtype], self.scale)
        self.pools, self.table, self.contexts = coded_pools(rng, hkv, d, bs, kv, junk=junk, scales=scales)
        self.cache = spork.make_kvq(**self.pools)
        rows = sum(new)
        wide = torch.from_numpy(rng.standard_normal((rows + spare_rows, hq * d + gap)).astype(np.float32) * gain).to(dtype).cuda()
        self.q = wide[:, :hq * d].unflatten(1, (hq, d))
        self.rows = rows
        self.row_off = torch.tensor(np.cumsum([0] + list(new)), dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(list(kv), dtype=torch.int32, device="cuda")
        self.out = torch.full((rows + spare_rows, hq, d), 7.5, dtype=dtype, device="cuda")
        self.lse = torch.full((rows + spare_rows, hq), 7.5, dtype=F32, device="cuda")
        self.ws = torch.full((spork.spork_chunk_workspace_bytes(self.shape, len(new), rows + spare_rows) // 4,), float("nan"),
                             dtype=F32, device="cuda")

    def run(self, lse=True):
        spork.spork_kvq_attn(self.shape, self.q, self.cache, self.table, self.row_off, self.kv_len, self.out, self.lse if lse else None,
                             self.ws)


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF16, 4, 1, 128), (BF16, 2, 2, 64), (F32, 2, 1, 64), (F32, 3, 3, 128)])
def test_single_tokens_around_every_edge(dtype, hq, hkv, d, bs):
    Case(dtype, hq, hkv, d, bs, [1] * len(EDGES), EDGES).run_and_check("single tokens")


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF16, 8, 1, 128), (BF16, 3, 3, 64), (F32, 4, 2, 64), (F32, 2, 2, 128)])
def test_whole_prompts_around_every_edge(dtype, hq, hkv, d, bs):
    Case(dtype, hq, hkv, d, bs, EDGES, EDGES, gap=8 * hkv).run_and_check("whole prompts")


@pytest.mark.parametrize("dtype,hq,hkv,d,bs,new,kv", [
    (BF16, 8, 2, 128, 16, [5, 0, 64, 1, 0, 33, 2], [900, 77, 64, 1, 0, 500, 31]),
    (BF16, 7, 1, 128, 32, [40, 1, 300], [41, 1000, 700]),
    (BF16, 28, 4, 128, 16, [37, 73], [500, 73]),
    (BF16, 16, 1, 64, 16, [16, 17, 100], [300, 17, 101]),
    (BF16, 5, 5, 64, 32, [260, 513], [1000, 513]),
    (BF16, 256, 1, 64, 16, [3, 1], [50, 400]),
    (BF16, 200, 2, 128, 32, [4], [200]),
    (F32, 8, 2, 128, 16, [5, 0, 64, 1, 33], [300, 77, 64, 1, 200]),
    (F32, 7, 1, 64, 32, [40, 1, 90], [41, 700, 300]),
    (F32, 256, 1, 64, 16, [2, 1], [40, 100]),
])
def test_mixed_batches(dtype, hq, hkv, d, bs, new, kv):
    Case(dtype, hq, hkv, d, bs, new, kv, gap=16).run_and_check("mixed")


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("dtype,hq,hkv,d,new,kv", [
    (BF16, 8, 2, 128, [1, 3, 40], [700, 333, 90]), (BF16, 4, 4, 64, [1, 200], [900, 260]), (F32, 4, 2, 64, [1, 20], [300, 90]),
    (F32, 2, 1, 128, [2, 40], [200, 44]), (BF16, 8, 1, 128, [60, 33], [400, 290])])
def test_scales_far_apart(dtype, hq, hkv, d, bs, new, kv):
    """Blocks whose values are 2^12 apart: a scale of the wrong block, head, or of values for keys shows."""
    Case(dtype, hq, hkv, d, bs, new, kv, scales=(111, 123), scale=0.02).run_and_check("scales")


@pytest.mark.parametrize("low,high", ((27, 30), (245, 248)))
@pytest.mark.parametrize("dtype", (BF16, F32))
def test_values_at_the_ends_of_the_scales(dtype, low, high):
    """Values at the smallest and largest scales that a write makes, under keys of ordinary ones. (Smaller: the outputs are
    small; larger: the sum of a row's values stays below the largest number.)"""
    c = Case(dtype, 4, 2, 128, 16, [1, 7], [60, 30])
    rng = np.random.default_rng(low)
    e = rng.integers(low, high, c.pools["v_scale"].shape).astype(np.uint8)
    codes = c.pools["v_codes"].cpu().numpy()
    codes[codes & 127 > 80] -= 40
    c.pools["v_codes"].copy_(torch.from_numpy(codes))
    c.pools["v_scale"].copy_(torch.from_numpy(e))
    table, contexts = c.table.cpu().numpy(), []
    for s, length in enumerate(c.kv):
        ids = table[s, :blocks_of(length, 16)]
        v = VALUES[codes[ids]] * 2.0 ** (e[ids].astype(np.float64) - 127)[:, :, None, None]
        contexts.append((c.contexts[s][0], torch.from_numpy(v.transpose(0, 3, 1, 2).reshape(-1, 2, 128)[:length].copy())))
    c.contexts = contexts
    c.run_and_check(f"scales {low}")


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("new,kv", [([20, 3], [5, 0]), ([300], [40]), ([1], [0]), ([64, 64], [63, 0]), ([700], [1]),
                                    ([257, 300], [0, 33])])
def test_rows_with_nothing_to_see(dtype, new, kv, d):
    """More rows than positions: the first rows lie before the sequence's start."""
    c = Case(dtype, 4, 2, d, 16, new, kv)
    c.run()
    torch.cuda.synchronize()
    o = []
    row = 0
    for (k, v), n in zip(c.contexts, new):
        hidden = max(0, n - k.shape[0])
        part = attention(c.q[row + hidden:row + n].cpu(), [(k, v)], [n - hidden], c.scale)
        o.append([torch.cat([torch.zeros(hidden, *x.shape[1:], dtype=x.dtype), x]) for x in part])
        o[-1][1][:hidden] = -math.inf
        row += n
    c.check("empty rows", ref=[torch.cat(x) for x in zip(*o)])


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("new,kv,hq,hkv", [
    ([1, 1], [30011, 70000], 8, 1),          # few rows, a long axis: every slice has a piece
    ([1], [66001], 4, 4),
    ([700], [9000], 8, 1),                   # tiles that a cut goes through
    ([1] * 40 + [257], [40 * i + 1 for i in range(40)] + [3001], 4, 1),
])
def test_tiles_split_over_slices(new, kv, hq, hkv, bs):
    c = Case(BF16, hq, hkv, 128, bs, new, kv, gain=3.0)
    c.run_and_check("split")
    first = (c.out.clone(), c.lse.clone())
    c.ws.fill_(float("inf"))
    c.out.fill_(7.5)
    c.lse.fill_(7.5)
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(first[0], c.out) and torch.equal(first[1], c.lse)


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("group", (8, 7))
@pytest.mark.parametrize("d", (64, 128))
def test_tiles_that_fill_a_workgroup(bs, group, d):
    """More than 128 packed rows per tile, contexts of one to ten stages, odd and even, whole and part."""
    new = [17, 20, 31, 32, 33, 19, 28, 36, 37, 64, 65, 18, 25, 29]
    kv = [17, 33, 63, 64, 65, 95, 97, 128, 130, 160, 190, 224, 288, 319]
    Case(BF16, group, 1, d, bs, new, kv, gain=2.0).run_and_check(f"groups of {group}")


@pytest.mark.parametrize("dtype,hq,hkv,d,bs,rows,length", [
    (BF16, 64, 8, 128, 16, 1024, 7011), (BF16, 64, 8, 64, 32, 1024, 7011), (BF16, 16, 2, 64, 16, 16, 9000),
    (BF16, 16, 2, 128, 32, 2, 20000), (F32, 16, 2, 64, 32, 20, 3000), (F32, 16, 2, 128, 16, 2, 3000)])
def test_every_stage_is_found(dtype, hq, hkv, d, bs, rows, length):
    """Rows that each seek one key, the keys in every stage of a context that is longer than several windows of the table:
    a stage left out, read twice or taken from elsewhere gives another token's values."""
    c = Case(dtype, hq, hkv, d, bs, [rows], [length], spare_rows=0)
    rng = np.random.default_rng(rows)
    keys, group = c.contexts[0][0], hq // hkv
    checked = list(range(rows)) if rows < 100 else [*range(32), *range(500, 532), *range(rows - 32, rows)]
    q = c.q.cpu().clone()
    for i, r in enumerate(checked):
        last = length - rows + r
        for h in range(hq):
            t = min((i * group + h % group) % (last // 32 + 1) * 32 + int(rng.integers(32)), last)
            q[r, h] = (4.0 * keys[t, h // group]).to(dtype)
    c.q.copy_(q)
    c.run()
    torch.cuda.synchronize()
    k, v = c.contexts[0]
    for r in checked:
        end = length - rows + r + 1
        ref = attention(q[r:r + 1], [(k[:end], v[:end])], [1], c.scale)
        o_tol, l_tol = bounds(dtype, *ref, c.scale, 32 + length // 16 + 64, d)  # 32 products in one, then stages, pieces and ways
        assert ((c.out[r:r + 1].double().cpu() - ref[0]).abs() <= o_tol).all(), r
        assert ((c.lse[r:r + 1].double().cpu() - ref[1]).abs() <= l_tol).all(), r


def test_every_code():
    """All codes but those that are no number, as keys and as values."""
    c = Case(F32, 2, 1, 128, 16, [1], [254 * 2], spare_rows=0, scales=(120, 121), scale=0.01)
    numbers = np.array([x for x in range(256) if x & 127 != 127], np.uint8)
    table = c.table[0].cpu().numpy()
    k, v = c.pools["k_codes"].cpu().numpy(), c.pools["v_codes"].cpu().numpy()
    x, y = np.zeros((508, 128), np.uint8), np.zeros((508, 128), np.uint8)
    for t in range(508):
        x[t], y[t] = np.roll(numbers, t)[:128], np.roll(numbers, 100 - t)[:128]
        k[table[t // 16], 0, t % 16], v[table[t // 16], 0, :, t % 16] = x[t], y[t]
    c.pools["k_codes"].copy_(torch.from_numpy(k))
    c.pools["v_codes"].copy_(torch.from_numpy(v))
    c.contexts = [tuple(torch.from_numpy(VALUES[z][:, None] * 2.0 ** -7) for z in (x, y))]
    c.run_and_check("codes")


@pytest.mark.parametrize("hq,hkv,d,bs,new,kv", [(8, 2, 128, 16, [1, 50, 300], [3000, 90, 700]), (4, 4, 64, 32, [1, 20], [900, 200])])
def test_the_same_values_in_bf16_pools(hq, hkv, d, bs, new, kv):
    """The other pools' attention over the values that the codes stand for: within both bounds of each other."""
    c = Case(BF16, hq, hkv, d, bs, new, kv, spare_rows=0, junk=0)
    c.run()
    k, v = ((c.pools[n + "_codes"].view(torch.float8_e4m3fn).float() * torch.exp2(c.pools[n + "_scale"].float() - 127)
             .nan_to_num(1, 1)[:, :, None, None]).to(BF16) for n in "kv")
    out, lse = c.out.clone(), c.lse.clone()
    spork.spork_chunk_attn(c.shape, c.q, k, v, c.table, c.row_off, c.kv_len, out, lse, c.ws)
    torch.cuda.synchronize()
    ref = c.reference()
    o_tol, l_tol = bounds(BF16, *ref, c.scale, max(kv), d)
    assert ((out.double() - c.out.double()).abs().cpu() <= 2 * o_tol).all()
    assert ((lse.double() - c.lse.double()).abs().cpu() <= 2 * l_tol).all()
    c.check("codes")


def test_many_sequences():
    """More sequences than threads of a workgroup, most without rows."""
    n = 1500
    new = [1 if i % 7 == 0 else 3 if i % 211 == 5 else 0 for i in range(n)]
    new[:300] = [0] * 300
    new[-64:] = [0] * 64
    kv = [(i * 13) % 90 + x for i, x in enumerate(new)]
    Case(BF16, 4, 2, 64, 16, new, kv).run_and_check("many")


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("scale,gain", [(0.0, 1.0), (-0.2, 1.0), (0.125, 30.0), (3.0, 4.0), (1e-30, 1.0)])
def test_softmax_scales(dtype, scale, gain):
    Case(dtype, 4, 2, 64, 16, [70, 1], [200, 90], scale=scale, gain=gain).run_and_check(f"scale {scale}")


@pytest.mark.parametrize("junk", [127, 255, 126, 254, 0])
@pytest.mark.parametrize("dtype,hq,new", [(BF16, 4, [33, 1, 7]), (F32, 4, [33, 1, 7]), (BF16, 8, [60, 1, 7])])
def test_unwritten_slots_may_hold_anything(dtype, junk, hq, new):
    Case(dtype, hq, 1, 128, 32, new, [70, 45, 7], junk=junk).run_and_check(f"junk {junk}")


def test_rows_that_are_no_number():
    """A query that holds a NaN spoils its own head's row and no other."""
    c = Case(BF16, 8, 2, 128, 16, [40, 1], [300, 90])
    c.run()
    torch.cuda.synchronize()
    want = (c.out.clone(), c.lse.clone())
    c.q[7, 3, 5] = float("nan")
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[7, 3]).all() and torch.isnan(c.lse[7, 3])
    for got, w in zip((c.out, c.lse), want):
        got[7, 3] = w[7, 3]
        assert torch.equal(got, w)


def test_entries_out_of_range_are_clamped():
    """Bad tables, offsets and lengths: no access out of bounds, and the sound sequences' rows are right."""
    c = Case(BF16, 4, 1, 128, 16, [5, 5, 5], [100, 100, 100])
    ref = c.reference()
    c.table[1] = torch.tensor([1 << 30, -5, 2 ** 31 - 1, -2 ** 31, 1 << 20, 9999, -1], dtype=torch.int32)
    c.run()
    torch.cuda.synchronize()
    want = c.out.clone()
    c.out.fill_(7.5)
    c.kv_len[1] = 1 << 30
    c.row_off[3] = 1 << 30  # the last sequence takes the spare rows too
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:5], want[:5])
    o_tol, _ = bounds(BF16, *ref, c.scale, 100, 128)
    assert ((want[:5].double().cpu() - ref[0][:5]).abs() <= o_tol[:5]).all()
    c.kv_len[:] = -3
    c.row_off[:] = torch.tensor([9, -4, 1 << 30, -1 << 31], dtype=torch.int32)
    c.run()
    torch.cuda.synchronize()


def test_no_lse_no_rows_no_sequences():
    c = Case(BF16, 4, 1, 128, 16, [9, 40], [50, 40])
    c.run()
    torch.cuda.synchronize()
    want = c.out.clone()
    c.out.fill_(7.5)
    c.lse.fill_(7.5)
    c.run(lse=False)
    torch.cuda.synchronize()
    assert torch.equal(c.out, want) and (c.lse == 7.5).all()
    c.out.fill_(7.5)
    c.row_off.zero_()
    c.run()
    torch.cuda.synchronize()
    assert (c.out == 7.5).all()
    spork.spork_kvq_attn(c.shape, c.q[:0], c.cache, c.table, c.row_off, c.kv_len, c.out[:0], c.lse[:0], None)
    spork.spork_kvq_attn(c.shape, c.q, c.cache, c.table[:0], c.row_off[:1], c.kv_len[:0], c.out, c.lse, None)
    torch.cuda.synchronize()
    assert (c.out == 7.5).all()


def test_two_streams():
    cases = [Case(BF16, 4, 1, 128, 16, [90, 1], [300, 500], seed=1), Case(F32, 4, 2, 64, 32, [9, 1], [300, 500], seed=2)]
    torch.cuda.synchronize()
    for c in cases:
        with torch.cuda.stream(torch.cuda.Stream()):
            c.run()
    for c in cases:
        c.check("stream")


def test_captured_calls_follow_the_lengths():
    """One graph; lengths, offsets, tables, codes and scales change between replays, and eager calls run in between."""
    cases = [Case(BF16, 8, 2, 128, 16, new, kv, seed=i, spare_rows=128 - sum(new)) for i, (new, kv) in enumerate(
        [([1, 1, 1], [400, 90, 3]), ([100, 1, 0], [130, 500, 64]), ([0, 60, 17], [5, 60, 480]), ([0, 0, 0], [1, 2, 3])])]
    most = max(c.table.shape[1] for c in cases)
    blocks = max(c.pools["k_scale"].shape[0] for c in cases)
    live = cases[0]
    hold = dict(q=torch.empty_like(live.q), table=torch.zeros(3, most, dtype=torch.int32, device="cuda"), row_off=live.row_off.clone(),
                kv_len=live.kv_len.clone())
    pools = {n: t.new_zeros(blocks, *t.shape[1:]) for n, t in live.pools.items()}
    cache = spork.make_kvq(**pools)
    out, lse, ws = live.out.clone(), live.lse.clone(), live.ws.clone()

    def fill(c):
        for name in ("q", "row_off", "kv_len"):
            hold[name].copy_(getattr(c, name))
        for n, t in c.pools.items():
            pools[n][:t.shape[0]] = t
        hold["table"][:, :c.table.shape[1]] = c.table
        out.fill_(7.5)
        lse.fill_(7.5)

    def run():
        spork.spork_kvq_attn(live.shape, hold["q"], cache, hold["table"], hold["row_off"], hold["kv_len"], out, lse, ws)

    fill(cases[0])
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for r, c in enumerate(cases + cases[:2]):
        fill(c)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.out.copy_(out)
        c.lse.copy_(lse)
        c.check(f"replay {r}")
        c.run()  # eager, on its own buffers
        torch.cuda.synchronize()
        assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


@pytest.mark.parametrize("new", ([1, 3], [300, 1]))
def test_blocks_past_4_gib(new):
    """Blocks whose codes begin beyond 2^32 bytes."""
    c = Case(BF16, 8, 8, 128, 32, new, [400, 333], seed=6)
    nb, used = 135000, c.pools["k_scale"].shape[0]  # 32 KiB a block
    big = {n: torch.zeros((nb, *t.shape[1:]), dtype=torch.uint8, device="cuda") for n, t in c.pools.items()}
    for n, t in c.pools.items():
        big[n][nb - used:] = t
    spork.spork_kvq_attn(c.shape, c.q, spork.make_kvq(**big), c.table + (nb - used), c.row_off, c.kv_len, c.out, c.lse, c.ws)
    c.check("past 4 GiB")
    say("  blocks past 4 GiB")
