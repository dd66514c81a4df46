"""Block tables and slots built on the GPU from request lengths
(spork_tables_step) against a sequential model of the same rules, bit for bit:
tables, references, free queue, slots, copies. With the host block manager the
same appends and forks give the same tables. Plus the batched block copy."""
import random

import numpy as np
import pytest
import torch

from oracle.kv import copy_block_prefix
from paged_cases import TablesModel, blocks_of
from gpu_cases import say
from paper_2607_03333_amd import spork

pytestmark = pytest.mark.gpu


class Device:
    """Tables on the GPU with their outputs, poisoned before every step."""

    def __init__(self, n, num_blocks, bs, max_blocks, order=None):
        ints = lambda *m: torch.full(m, -77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.n, self.bs, self.nb = n, bs, num_blocks
        self.table, self.held, self.refs = ints(n, max_blocks), ints(n), ints(num_blocks)
        self.ring, self.queue = ints(num_blocks), ints(2)
        self.t = spork.make_tables(bs, self.table, self.held, self.refs, self.ring, self.queue)
        spork.spork_tables_init(self.t, None if order is None else torch.as_tensor(order, dtype=torch.int32).cuda())
        self.ws = torch.full((spork.spork_tables_workspace_bytes(self.t),), 0x5A, dtype=torch.uint8, device="cuda")
        spork.spork_tables_workspace_clear(self.t, self.ws)
        self.lens, self.new, self.parents = ints(n), ints(n), ints(n)
        self.row_off, self.kv_len, self.copies, self.n_copies, self.status = ints(n + 1), ints(n), ints(n, 3), ints(1), ints(1)

    def sized(self, max_tokens):
        self.slots = torch.full((max_tokens,), -77, dtype=torch.int64, device="cuda")
        self.positions = torch.full((max_tokens,), -77, dtype=torch.int32, device="cuda")

    def set(self, lens, new, parents):
        for t, x in ((self.lens, lens), (self.new, new), (self.parents, parents or [-1] * self.n)):
            t.copy_(torch.tensor(x, dtype=torch.int32))

    def launch(self, forks=True):
        spork.spork_tables_step(self.t, self.lens, self.new, self.parents if forks else None, self.slots, self.positions,
                                self.row_off, self.kv_len, self.copies, self.n_copies, self.status, self.ws)

    def step(self, lens, new, parents, max_tokens):
        self.set(lens, new, parents)
        self.sized(max_tokens)
        for t in (self.row_off, self.kv_len, self.copies, self.n_copies, self.status):
            t.fill_(-77)
        self.launch(parents is not None)
        torch.cuda.synchronize()

    def check(self, model, want, max_tokens):
        status, slots, positions, off, kv_len, copies = want
        assert self.status.item() == status
        pad = [-1] * (max_tokens - len(slots))
        assert self.slots.tolist() == slots + pad and self.positions.tolist() == positions + pad
        assert self.row_off.tolist() == off and self.kv_len.tolist() == kv_len
        assert self.n_copies.item() == len(copies)
        assert [tuple(c) for c in self.copies.tolist()[:len(copies)]] == copies
        assert all(c == [-77] * 3 for c in self.copies.tolist()[len(copies):])
        assert self.held.tolist() == [len(r) for r in model.rows]
        table = self.table.tolist()
        assert all(table[s][:len(r)] == r for s, r in enumerate(model.rows))
        assert self.refs.tolist() == model.refs
        front, count = self.queue.tolist()
        ring = self.ring.tolist()
        assert [ring[(front + i) % self.nb] for i in range(count)] == model.queue


def _random_steps(rnd, n, bs, max_blocks, model, steps):
    """Steps of a batch that rolls back, ends, forks and appends; some do not fit."""
    lens = [0] * n
    for _ in range(steps):
        parents, before, new = [-1] * n, list(lens), [0] * n
        for s in range(n):
            what = rnd.random()
            if what < 0.1:
                before[s] = 0
            elif what < 0.4:
                before[s] = rnd.randint(max(0, lens[s] - 2 * bs), lens[s])
            room = max_blocks * bs - before[s]
            new[s] = rnd.choice((0, 1, 1, rnd.randint(0, 3 * bs)))
            if rnd.random() < 0.02:
                new[s] = room + rnd.randint(0, 2)
            new[s] = min(new[s], room) if rnd.random() < 0.9 else new[s]
        mains = [s for s in range(n) if rnd.random() < 0.5]
        for s in range(n):
            if mains and s not in mains and rnd.random() < 0.4:
                p = rnd.choice(mains)
                parents[s], before[s] = p, rnd.randint(max(0, lens[p] - bs), lens[p])
                new[s] = min(rnd.randint(0, 2 * bs), max_blocks * bs - before[s])
        yield before, new, parents
        if model.last == 0:
            lens = [a + b for a, b in zip(before, new)]


@pytest.mark.parametrize("n,num_blocks,bs,max_blocks,seed", [
    (1, 1, 16, 4, 0), (2, 7, 16, 3, 1), (5, 40, 4, 9, 2), (17, 150, 16, 12, 3), (33, 120, 1, 6, 4), (70, 900, 32, 11, 5),
    (300, 2000, 16, 7, 6), (1100, 9000, 8, 9, 7)])
def test_steps_match_the_model(n, num_blocks, bs, max_blocks, seed):
    rnd = random.Random(seed)
    order = rnd.sample(range(num_blocks), num_blocks)
    model = TablesModel(n, num_blocks, bs, max_blocks, order)
    model.last = 0
    dev = Device(n, num_blocks, bs, max_blocks, order)
    codes = {}
    for before, new, parents in _random_steps(rnd, n, bs, max_blocks, model, 14):
        max_tokens = max(0, sum(new) + rnd.choice((0, 0, 1, 300, -1 if rnd.random() < 0.2 else 0)))
        want = model.step(before, new, parents, max_tokens)
        model.last = want[0]
        dev.step(before, new, parents, max_tokens)
        dev.check(model, want, max_tokens)
        codes[want[0]] = codes.get(want[0], 0) + 1
    say(f"  tables n={n} blocks={num_blocks} bs={bs}: steps by status {codes}")
    assert codes.get(0, 0) >= 1
    # the workspace is as it was cleared
    words = 32 // 4 + 3 * num_blocks
    assert not control_words(dev.ws, words).any()


def control_words(ws, words):
    return ws[:4 * words].view(torch.int32)[[i for i in range(words) if not 2 <= i < 8]]


def test_long_rows_and_whole_batches_end():
    """A prompt of 70,000 tokens, its forks, and everything ending at once, in table order."""
    bs, n = 16, 6
    per = blocks_of(70000 + 64, bs)
    nb = per + 5 * 40 + 400
    order = np.random.default_rng(3).permutation(nb).tolist()
    model, dev = TablesModel(n, nb, bs, per, order), Device(n, nb, bs, per, order)
    steps = [([0] * n, [70000, 0, 0, 0, 0, 33], [-1] * n), ([70000, 69999, 70000, 16, 0, 33], [1, 5, 0, 40, 7, 0], [-1, 0, 0, 0, 0, -1]),
             ([69000, 70004, 70000, 56, 7, 0], [1, 1, 1, 1, 1, 0], [-1] * n), ([0] * n, [0] * n, [-1] * n)]
    for lens, new, parents in steps:
        want = model.step(lens, new, parents, 70100)
        assert want[0] == 0
        dev.step(lens, new, parents, 70100)
        dev.check(model, want, 70100)
    assert sorted(model.queue) == list(range(nb))


def test_probes_that_fork_again_where_they_were():
    """Rows that give up and take over the same entries in one step, with a parent that grows, is rolled back below
    them or ends, and steps that are refused in between."""
    bs, nb, n, most = 16, 700, 7, 40
    order = np.random.default_rng(9).permutation(nb).tolist()
    model, dev = TablesModel(n, nb, bs, most, order), Device(n, nb, bs, most, order)
    fork = [-1, 0, 0, -1, 3, 3, 3]
    steps = [([0] * n, [333, 0, 0, 100, 0, 0, 0], [-1] * n), ([333, 333, 320, 100, 100, 99, 96], [9, 30, 8, 1, 1, 1, 1], fork),
             ([340, 338, 338, 101, 101, 101, 50], [3, 30, 50, 1, 0, 12, 1], fork), ([340, 340, 16, 101, 101, 101, 50], [800, 0, 0, 0, 0, 0, 0], fork),
             ([20, 343, 343, 90, 102, 102, 0], [5, 1, 1, 0, 0, 0, 0], fork), ([0, 25, 25, 0, 90, 16, 90], [0, 3, 3, 0, 3, 3, 3], fork),
             ([0, 28, 28, 0, 93, 19, 93], [0, 1, 1, 0, 1, 1, 1], [-1] * n), ([0] * n, [0] * n, [-1] * n)]
    codes = []
    for lens, new, parents in steps:
        want = model.step(lens, new, parents, 500)
        dev.step(lens, new, parents, 500)
        dev.check(model, want, 500)
        codes.append(want[0])
    assert codes == [0, 0, 0, -4, 0, 0, 0, 0] and sorted(model.queue) == list(range(nb))


def test_refused_steps_change_nothing():
    n, nb, bs, most = 4, 12, 16, 4
    model, dev = TablesModel(n, nb, bs, most), Device(n, nb, bs, most)
    good = ([0] * n, [20, 5, 0, 16], None)
    dev.step(*good, 64)
    dev.check(model, model.step(*good, 64), 64)
    stay = [20, 5, 0, 16]
    refused = [
        (-1, [-1, 5, 0, 16], [1, 0, 0, 0], None), (-1, stay, [0, -1, 0, 0], None), (-1, [33, 5, 0, 16], [0] * 4, None),
        (-4, stay, [45, 0, 0, 0], None), (-4, stay, [0, 0, 65, 0], None), (-2, stay, [30, 30, 60, 40], None),
        (-1, stay, [0] * 4, [0, -1, -1, -1]), (-1, stay, [0] * 4, [-1, 4, -1, -1]), (-1, stay, [0] * 4, [-1, 0, 1, -1]),
        (-1, [20, 33, 0, 16], [0] * 4, [-1, 0, -1, -1]), (-4, [20, 17, 0, -2], [45, 9, 0, 0], [-1, 0, -1, -1]),
        (-4, stay, [30, 0, 0, 0], None)]
    for code, lens, new, parents in refused:
        most_tokens = {30: 29, 160: 160}.get(sum(new), 64)
        want = model.step(lens, new, parents, most_tokens)
        assert want[0] == code, (lens, new, parents)
        dev.step(lens, new, parents, most_tokens)
        dev.check(model, want, most_tokens)
    # entries outside the pool, of rows that the step touches, and a queue that is none
    for spoil, restore in ((lambda: dev.table[0, 1].fill_(nb), lambda: dev.table[0, 1].fill_(1)),
                           (lambda: dev.table[0, 1].fill_(-1), lambda: dev.table[0, 1].fill_(1)),
                           (lambda: dev.queue[1].fill_(nb + 1), lambda: dev.queue[1].fill_(8)),
                           (lambda: dev.queue[0].fill_(-1), lambda: dev.queue[0].fill_(4))):
        spoil()
        dev.step([5, 5, 0, 16], [1, 0, 0, 0], None, 64)
        assert dev.status.item() == -1 and dev.row_off.tolist() == [0] * 5 and (dev.slots == -1).all()
        restore()
        dev.check(model, (-1, [], [], [0] * 5, [0] * 4, []), 64)
    dev.step([20, 5, 0, 16], [1, 1, 1, 1], None, 4)
    dev.check(model, model.step([20, 5, 0, 16], [1, 1, 1, 1], None, 4), 4)


def test_same_tables_as_the_host_block_manager():
    bs, nb, n = 16, 200, 6
    order = np.random.default_rng(5).permutation(nb)
    cache = spork.spork_cache_create(nb, bs, order)
    try:
        dev = Device(n, nb, bs, 30, order)
        seqs = [spork.spork_seq_new(cache) for _ in range(2)]
        slots, _ = spork.spork_seq_append_batch(cache, seqs, [100, 37])
        dev.step([0] * n, [100, 37, 0, 0, 0, 0], None, 200)
        assert dev.slots.tolist()[:137] == slots.tolist()
        seqs += [spork.spork_fork(cache, seqs[p]) for p in (0, 0, 1, 0)]
        new = [1, 9, 8, 50, 1, 3]
        slots, copies = spork.spork_seq_append_batch(cache, seqs, new)
        dev.step([100, 37, 100, 100, 37, 100], new, [-1, -1, 0, 0, 1, 0], 200)
        assert dev.slots.tolist()[:72] == slots.tolist()
        assert [tuple(c) for c in dev.copies.tolist()[:dev.n_copies.item()]] == copies
        assert copies
        table = dev.table.tolist()
        for s, q in enumerate(seqs):
            got = spork.spork_block_table(cache, q).tolist()
            assert table[s][:dev.held[s].item()] == got
        front, count = dev.queue.tolist()
        ring = dev.ring.tolist()
        assert [ring[(front + i) % nb] for i in range(count)] == spork.spork_free_blocks(cache).tolist()
        assert dev.refs.tolist() == [spork.spork_refcount(cache, b) for b in range(nb)]
    finally:
        spork.spork_cache_destroy(cache)


def test_captured_steps_follow_the_lengths():
    """One graph, replayed with other lengths each time; eager steps and other work between replays."""
    bs, nb, n = 16, 300, 9
    model, dev = TablesModel(n, nb, bs, 12), Device(n, nb, bs, 12)
    dev.sized(400)
    dev.set([0] * n, [0] * n, [-1] * n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dev.launch()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    model.step([0] * n, [0] * n, [-1] * n, 400)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dev.launch()
    steps = [([0] * n, [40, 17, 0, 16, 1, 0, 0, 0, 0], [-1] * n),
             ([40, 17, 40, 16, 1, 39, 17, 0, 0], [1, 1, 8, 9, 0, 30, 2, 5, 0], [-1, -1, 0, -1, -1, 0, 1, -1, -1]),
             ([38, 18, 48, 20, 1, 69, 19, 0, 0], [3, 1, 1, 1, 1, 1, 1, 1, 1], [-1] * n),
             ([0] * n, [0] * n, [-1] * n), ([0] * n, [11] * n, [-1] * n)]
    for lens, new, parents in steps:
        want = model.step(lens, new, parents, 400)
        dev.set(lens, new, parents)
        dev.copies.fill_(-77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        dev.check(model, want, 400)


@pytest.mark.parametrize("dtype,hkv,d,bs", [(torch.float32, 2, 64, 16), (torch.bfloat16, 4, 128, 16), (torch.bfloat16, 1, 64, 32),
                                            (torch.float32, 3, 20, 5), (torch.bfloat16, 2, 8, 1)])
def test_copy_batch(dtype, hkv, d, bs):
    gen = torch.Generator().manual_seed(bs + d)
    nb = 20
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    k = torch.randint(-30000, 30000, (nb, hkv, bs, d), generator=gen).to(bits)
    v = torch.randint(-30000, 30000, (nb, hkv, d, bs), generator=gen).to(bits)
    entries = [(3, 7, 1), (0, 11, bs), (3, 2, max(1, bs - 1)), (nb, 4, 1), (5, nb, 1), (-1, 4, 1), (5, -3, 1), (6, 6, 1), (6, 8, 0),
               (6, 8, bs + 1), (6, 8, -1), (19, 1, max(1, bs // 2)), (12, 13, bs)]
    real = [e for e in entries[:-1] if 0 <= e[0] < nb and 0 <= e[1] < nb and e[0] != e[1] and 0 < e[2] <= bs]
    dk, dv = k.cuda(), v.cuda()
    shape = spork.make_shape(hkv, hkv, d, bs, spork.SPORK_DTYPE_BF16 if dtype == torch.bfloat16 else spork.SPORK_DTYPE_F32, 1.0)
    copies = torch.tensor(entries, dtype=torch.int32, device="cuda")
    count = torch.tensor([len(entries) - 1], dtype=torch.int32, device="cuda")  # the last entry is not counted
    spork.spork_kv_copy_batch(shape, dk, dv, nb, copies, count)
    for src, dst, m in real:
        copy_block_prefix(k, v, src, dst, m)
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)
    count.fill_(1 << 30)  # more than the list holds: the whole list
    spork.spork_kv_copy_batch(shape, dk, dv, nb, copies, count)
    for src, dst, m in real + [entries[-1]]:
        copy_block_prefix(k, v, src, dst, m)
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)
    count.fill_(-1)
    spork.spork_kv_copy_batch(shape, dk, dv, nb, copies, count)
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)


def test_a_queue_of_other_numbers_stays_inside_the_buffers():
    """Free-queue entries that are no blocks: they come out as they went in, and nothing beside the references changes."""
    for n, max_tokens in ((3, 200), (70, 6000)):
        nb, bs, most = 64, 16, 8
        ints = lambda *m: torch.full(m, -77, dtype=torch.int32, device="cuda")  # noqa: E731
        guarded = ints(nb + 2 * 4096)  # references in the middle
        dev = Device(n, nb, bs, most)
        dev.refs = guarded[4096:4096 + nb]
        dev.t = spork.make_tables(bs, dev.table, dev.held, dev.refs, dev.ring, dev.queue)
        spork.spork_tables_init(dev.t)
        odd = [-1, nb, nb + 4000, -4000, 5, 6, -(1 << 20), nb + 1]
        dev.ring[:8] = torch.tensor(odd, dtype=torch.int32)
        dev.step([0] * n, [100, 20] + [0] * (n - 2), None, max_tokens)
        assert dev.status.item() == 0 and dev.queue.tolist() == [9, nb - 9]
        assert dev.table[0, :7].tolist() == odd[:7] and dev.table[1, :2].tolist() == [odd[7], 8]
        assert dev.slots[:100].tolist() == [odd[i // bs] * bs + i % bs for i in range(100)]
        assert dev.refs.tolist() == [1 if i in (5, 6, 8) else 0 for i in range(nb)]
        assert (guarded[:4096] == -77).all() and (guarded[4096 + nb:] == -77).all()
        # rows with such entries are refused when they are released
        dev.step([0] * n, [0] * n, [-1] * n, max_tokens)
        assert dev.status.item() == spork.SPORK_E_INVAL and dev.refs.tolist() == [1 if i in (5, 6, 8) else 0 for i in range(nb)]
        assert (guarded[:4096] == -77).all() and (guarded[4096 + nb:] == -77).all()


def test_steps_of_one_launch_and_of_more_agree():
    """Steps at the rows, entries of a row and new-token places that the single launch takes, and at one more of each."""
    for n, most, extra in ((16, 9, 0), (17, 9, 0), (16, 9, 1), (3, 512, 0), (3, 513, 0), (1, 9, 0)):
        rnd = random.Random(n)
        nb, bs = 600, 16
        model, dev = TablesModel(n, nb, bs, most), Device(n, nb, bs, most)
        model.last = 0
        for before, new, parents in _random_steps(rnd, n, bs, most, model, 8):
            want = model.step(before, new, parents, 4096 + extra)
            model.last = want[0]
            dev.step(before, new, parents, 4096 + extra)
            dev.check(model, want, 4096 + extra)
        assert not control_words(dev.ws, 32 // 4 + 3 * nb).any()


@pytest.mark.parametrize("n,most", [(16, 512), (16, 513)])
def test_long_rows_of_one_launch(n, most):
    """As many entries as the single launch takes, all forked, rolled back and ended at once."""
    bs, nb = 4, 16 * 520
    order = np.random.default_rng(most).permutation(nb).tolist()
    model, dev = TablesModel(n, nb, bs, most, order), Device(n, nb, bs, most, order)
    lens = [0] * n
    for _ in range(4):
        new = [min(520, most * bs - x) if s % 4 < 2 else 0 for s, x in enumerate(lens)]
        new = [x if sum(new[:s + 1]) <= 4000 else 0 for s, x in enumerate(new)]
        want = model.step(lens, new, [-1] * n, 4096)
        assert want[0] == 0
        dev.step(lens, new, [-1] * n, 4096)
        dev.check(model, want, 4096)
        lens = [a + b for a, b in zip(lens, new)]
    for lens2, parents in (([lens[s - s % 4] - s % 4 if s % 4 > 1 else lens[s] for s in range(n)],
                            [s - s % 4 if s % 4 > 1 else -1 for s in range(n)]), ([0] * n, [-1] * n)):
        want = model.step([max(x, 0) for x in lens2], [0] * n, parents, 4096)
        assert want[0] == 0
        dev.step([max(x, 0) for x in lens2], [0] * n, parents, 4096)
        dev.check(model, want, 4096)


@pytest.mark.parametrize("n", (3, 20))
def test_slots_past_32_bits(n):
    """Slots of blocks at the end of a pool of 2^27 + 9 blocks of 64 tokens, and behind its wrap."""
    nb, bs, most = (1 << 27) + 9, 64, 8
    dev = Device(n, nb, bs, most)
    dev.queue[0] = nb - 3
    dev.step([0] * n, [200, 70] + [0] * (n - 2), None, 300)
    assert dev.status.item() == 0 and dev.queue.tolist() == [3, nb - 6]
    rows = [[nb - 3, nb - 2, nb - 1, 0], [1, 2]]
    assert [dev.table[s, :len(r)].tolist() for s, r in enumerate(rows)] == rows
    want = [rows[0][i // bs] * bs + i % bs for i in range(200)] + [rows[1][i // bs] * bs + i % bs for i in range(70)]
    assert dev.slots.tolist() == want + [-1] * 30 and max(want) > 1 << 32
    assert dev.refs.sum().item() == 6
