"""A server's steps over the cache of 8-bit codes: tables and slots, the copies of
shared blocks, the new tokens' rows normed, rotated and coded, the attention, and
the accept whose lengths the next step starts from, eagerly and as one replayed
graph, against a cache that is kept token by token in Python. Beside it the bf16
cache behind spork_qk_rope."""
import math

import numpy as np
import pytest
import torch

from gpu_cases import say
from paged_cases import TablesModel, attention, bounds
from paper_2607_03333_amd import spork
from rows_cases import PoolModel, same_codes, to_f64, turn_bound, turned
from test_gpu_paged_run import BF16, F32, SPORK, STEPS, captured

pytestmark = pytest.mark.gpu
EPS = 1e-6


class Server:
    def __init__(self, dtype, hq, hkv, d, bs, n, blocks, max_blocks, most, seed, rotary, interleaved=False, coded=True):
        ints = lambda *m: torch.zeros(*m, dtype=torch.int32, device="cuda")  # noqa: E731
        self.rng = np.random.default_rng(seed)
        self.dtype, self.n, self.most, self.hq, self.hkv, self.d, self.bs, self.coded = dtype, n, most, hq, hkv, d, bs, coded
        self.scale = float(np.float32(1.0 / math.sqrt(d)))
        self.shape = spork.make_shape(hq, hkv, d, bs, SPORK[dtype], self.scale)
        self.table = ints(n, max_blocks)
        self.t = spork.make_tables(bs, self.table, ints(n), ints(blocks), ints(blocks), ints(2))
        order = self.rng.permutation(blocks).astype(np.int32)
        spork.spork_tables_init(self.t, torch.from_numpy(order).cuda())
        self.model = TablesModel(n, blocks, bs, max_blocks, order)
        self.tables_ws = torch.empty(spork.spork_tables_workspace_bytes(self.t), dtype=torch.uint8, device="cuda")
        spork.spork_tables_workspace_clear(self.t, self.tables_ws)
        self.chunk_ws = torch.full((spork.spork_chunk_workspace_bytes(self.shape, n, most) // 4,), float("nan"), device="cuda")
        self.lens, self.new, self.parents = ints(n), ints(n), ints(n)
        self.slots = torch.zeros(most, dtype=torch.int64, device="cuda")
        self.positions, self.row_off, self.kv_len = ints(most), ints(n + 1), ints(n)
        self.copies, self.n_copies, self.status = ints(n, 3), ints(1), ints(1)
        self.rows = torch.zeros(most, (hq + 2 * hkv) * d, dtype=dtype, device="cuda")
        part = lambda a, h: self.rows[:, a * d:(a + h) * d].unflatten(1, (h, d))  # noqa: E731
        self.q, self.k_new, self.v_new = part(0, hq), part(hq, hkv), part(hq + hkv, hkv)
        self.q_out = torch.zeros(most, hq, d, dtype=dtype, device="cuda")
        self.out = torch.zeros(most, hq, d, dtype=dtype, device="cuda")
        self.lse = torch.zeros(most, hq, dtype=F32, device="cuda")
        self.inv_freq, self.magnitude = spork.spork_rope_frequencies(
            rotary, 10000.0, spork.spork_rope_scaling(spork.SPORK_ROPE_SCALE_PARTS, 64, 4.0, 32.0, 1.0))
        self.interleaved = interleaved
        layout = spork.SPORK_ROPE_INTERLEAVED if interleaved else spork.SPORK_ROPE_HALF
        self.rope = spork.make_rope(torch.from_numpy(self.inv_freq).cuda(), layout, self.magnitude)
        self.weights = [(1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(seed + i))).to(dtype).cuda() for i in (0, 1)]
        self.norm = spork.make_qk_norm(*self.weights, EPS)
        if coded:
            codes, scale = np.full((blocks, hkv, bs, d), 127, np.uint8), np.full((blocks, hkv), 200, np.uint8)
            gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
            self.pools = dict(k_codes=gpu(codes), v_codes=gpu(codes.swapaxes(2, 3)), k_scale=gpu(scale), v_scale=gpu(scale))
            self.cache = spork.make_kvq(**self.pools)
            self.k, self.v = PoolModel(codes, scale), PoolModel(codes, scale)
        else:
            self.kp = torch.full((blocks, hkv, bs, d), float("nan"), dtype=dtype, device="cuda")
            self.vp = torch.full((blocks, hkv, d, bs), float("nan"), dtype=dtype, device="cuda")
            self.k_out = torch.zeros(most, hkv, d, dtype=dtype, device="cuda")
            self.v_ready = torch.zeros(most, hkv, d, dtype=dtype, device="cuda")

    def launch(self):
        spork.spork_tables_step(self.t, self.lens, self.new, self.parents, self.slots, self.positions, self.row_off, self.kv_len,
                                self.copies, self.n_copies, self.status, self.tables_ws)
        if self.coded:
            spork.spork_kvq_copy_batch(self.shape, self.cache, self.copies, self.n_copies)
            spork.spork_kvq_write(self.shape, self.cache, self.rope, self.norm, self.slots, self.positions, self.q, self.k_new, self.v_new,
                                  self.q_out)
            spork.spork_kvq_attn(self.shape, self.q_out, self.cache, self.table, self.row_off, self.kv_len, self.out, self.lse, self.chunk_ws)
            return
        blocks = self.kp.shape[0]
        spork.spork_kv_copy_batch(self.shape, self.kp, self.vp, blocks, self.copies, self.n_copies)
        spork.spork_qk_rope(self.shape, self.rope, self.norm, self.positions, self.q, self.k_new, self.q_out, self.k_out)
        spork.spork_kv_write(self.shape, self.kp, self.vp, blocks, self.slots, self.k_out, self.v_ready)
        spork.spork_chunk_attn(self.shape, self.q_out, self.kp, self.vp, self.table, self.row_off, self.kv_len, self.out, self.lse,
                               self.chunk_ws)

    def prepare(self, lens, new, parents):
        x = self.rng.standard_normal(tuple(self.rows.shape)) * np.exp(self.rng.uniform(-1, 1, (self.most, 1)))
        self.rows.copy_(torch.from_numpy(x.astype(np.float32)).to(self.dtype))
        if not self.coded:
            self.v_ready.copy_(self.v_new)
        for t in (self.out, self.lse, self.q_out):
            t.fill_(7.5)
        for t, y in ((self.lens, lens), (self.new, new), (self.parents, parents)):
            t.copy_(torch.tensor(y, dtype=torch.int32))
        torch.cuda.synchronize()

    def turned(self, x, which, positions):
        return turned(to_f64(x[:len(positions)]), to_f64(self.weights[which]), EPS, positions, self.inv_freq, self.magnitude, self.interleaved)

    def check(self, lens, new, parents, tag):
        torch.cuda.synchronize()
        status, slots, positions, off, kv, copies = self.model.step(lens, new, parents, self.most)
        rows, bs = len(slots), self.bs
        assert status == 0 == self.status.item() and self.slots[:rows].tolist() == slots and self.kv_len.tolist() == kv
        want, size = self.turned(self.q, 0, positions)
        assert (np.abs(to_f64(self.q_out[:rows]) - want) <= turn_bound(want, size, self.d, self.dtype == BF16)).all(), tag
        k, v = self.turned(self.k_new, 1, positions), to_f64(self.v_new[:rows])
        contexts = []
        if self.coded:
            for c in copies:
                self.k.copy(*c)
                self.v.copy(*c)
            row = 0
            while row < rows:
                m = 1
                while row + m < rows and slots[row + m] == slots[row] + m and slots[row + m] % bs:
                    m += 1
                self.k.write(slots[row] // bs, slots[row] % bs, k[0][row:row + m])
                self.v.write(slots[row] // bs, slots[row] % bs, v[row:row + m])
                row += m
            for name, p in (("k", self.k), ("v", self.v)):
                got = self.pools[name + "_codes"].cpu().numpy()
                assert same_codes(got if name == "k" else got.swapaxes(2, 3), p.codes), f"{tag}: codes of {name}"
                assert np.array_equal(self.pools[name + "_scale"].cpu().numpy(), p.scale), f"{tag}: scales of {name}"
            read = lambda p, b, n: torch.from_numpy(p.values(b, n))  # noqa: E731
            pools = (self.k, self.v)
        else:
            kp, vp = to_f64(self.kp), to_f64(self.vp)
            at = np.array(slots, np.int64)
            got = kp[at // bs, :, at % bs] if rows else k[0]
            assert (np.abs(got - k[0]) <= turn_bound(*k, self.d, self.dtype == BF16)).all(), f"{tag}: keys"
            read = lambda p, b, n: torch.from_numpy(p[b, :, :n].swapaxes(0, 1).copy())  # noqa: E731
            pools = (kp, vp.swapaxes(2, 3))
        for s in range(self.n):
            length, blocks = kv[s], self.model.rows[s]
            contexts.append(tuple(torch.cat([read(p, b, min(bs, length - i * bs)) for i, b in enumerate(blocks)]) if length else
                                  torch.zeros(0, self.hkv, self.d, dtype=torch.float64) for p in pools))
        out, lse, size, mass = attention(self.q_out[:rows].cpu(), contexts, new, self.scale)
        o_tol, l_tol = bounds(self.dtype, out, lse, size, mass, self.scale, max(kv) + 1, self.d)
        worst = ((self.out[:rows].double().cpu() - out).abs() / o_tol).max().item() if rows else 0.0
        worst_l = ((self.lse[:rows].double().cpu() - lse).abs() / l_tol).max().item() if rows else 0.0
        say(f"  {tag}: out at {worst:.2f}, lse at {worst_l:.2f} of the bound")
        assert worst <= 1 and worst_l <= 1
        for t in (self.out, self.lse, self.q_out):
            assert (t[rows:] == 7.5).all(), f"{tag}: rows behind the last"


HEADS = [(BF16, 8, 2, 128, 16, 128, False), (BF16, 4, 4, 64, 32, 32, True), (F32, 6, 2, 64, 16, 64, True), (BF16, 5, 1, 128, 32, 96, False)]


@pytest.mark.parametrize("coded", (True, False))
@pytest.mark.parametrize("graph", (False, True))
@pytest.mark.parametrize("dtype,hq,hkv,d,bs,rotary,interleaved", HEADS)
def test_a_batch_that_forks_rolls_back_and_ends(dtype, hq, hkv, d, bs, rotary, interleaved, graph, coded):
    s = Server(dtype, hq, hkv, d, bs, 6, 80, 24, 300, hq * d + bs, rotary, interleaved, coded)
    call = s.launch
    if graph:
        s.prepare([0] * 6, [0] * 6, [-1] * 6)
        call = captured(s.launch).replay
    for i, (lens, new, parents) in enumerate(STEPS):
        s.prepare(lens, new, parents)
        call()
        s.check(lens, new, parents, f"step {i}")


def test_two_servers_on_two_streams():
    servers = [Server(BF16, 8, 2, 128, 16, 6, 80, 24, 300, 21, 64), Server(F32, 4, 2, 64, 32, 6, 80, 24, 300, 22, 64)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, (lens, new, parents) in enumerate(STEPS):
        for s in servers:
            s.prepare(lens, new, parents)
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                s.launch()
        for s in servers:
            s.check(lens, new, parents, f"step {i}")


def test_a_refused_step_does_nothing():
    """More blocks asked for than are free: rows behind it have slot and position -1, and nothing is written."""
    s = Server(BF16, 4, 2, 64, 16, 3, 20, 16, 300, 5, 64)
    s.prepare([0] * 3, [100, 60, 0], [-1] * 3)
    s.launch()
    s.check([0] * 3, [100, 60, 0], [-1] * 3, "prompts")
    s.prepare([100, 60, 0], [20, 1, 200], [-1] * 3)
    before = [x.clone() for x in (*s.pools.values(), s.table, s.out, s.lse, s.q_out)]
    s.launch()
    torch.cuda.synchronize()
    assert s.status.item() == -2
    for x, y in zip((*s.pools.values(), s.table, s.out, s.lse, s.q_out), before):
        assert torch.equal(x, y)
    s.prepare([100, 60, 0], [20, 1, 100], [-1] * 3)
    s.launch()
    s.check([100, 60, 0], [20, 1, 100], [-1] * 3, "the one that fits")


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Launches go to the current device: with another one current, nothing is launched."""
    s = Server(BF16, 4, 2, 64, 16, 2, 9, 4, 8, 1, 64)
    s.prepare([0, 0], [3, 2], [-1, -1])
    stream = torch.cuda.current_stream()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    calls = (lambda: spork.spork_qk_rope(s.shape, s.rope, s.norm, s.positions, s.q, s.k_new, s.q_out, s.k_new, stream=stream),
             lambda: spork.spork_kvq_write(s.shape, s.cache, s.rope, s.norm, s.slots, s.positions, s.q, s.k_new, s.v_new, s.q_out,
                                           stream=stream),
             lambda: spork.spork_kvq_copy_batch(s.shape, s.cache, s.copies, s.n_copies, stream=stream),
             lambda: spork.spork_kvq_attn(s.shape, s.q_out, s.cache, s.table, s.row_off, s.kv_len, s.out, s.lse, s.chunk_ws, stream=stream))
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert (s.out == 7.5).all() and (s.q_out == 7.5).all()
