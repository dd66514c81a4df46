"""The steps whose lengths live on the GPU as a server runs them: tables and
slots, the copies of shared blocks, the writes of new keys and values, the
attention, and the accept whose lengths the next step starts from, eagerly and
as one replayed graph, against contexts that are kept token by token in Python."""
import math

import numpy as np
import pytest
import torch

from gpu_cases import say
from paged_cases import attention, bounds
from paper_2607_03333_amd import spork

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SPORK = {BF16: spork.SPORK_DTYPE_BF16, F32: spork.SPORK_DTYPE_F32}


class Server:
    """n rows over paged pools that hold NaN wherever nothing was written, static buffers for `most` new tokens, and
    the rows' contexts as lists of (key, value)."""

    def __init__(self, dtype, hq, hkv, d, bs, n, num_blocks, max_blocks, most, seed):
        ints = lambda *m: torch.zeros(*m, dtype=torch.int32, device="cuda")  # noqa: E731
        self.rng = np.random.default_rng(seed)
        self.dtype, self.n, self.most, self.hq, self.hkv, self.d = dtype, n, most, hq, hkv, d
        self.scale = float(np.float32(1.0 / math.sqrt(d)))
        self.shape = spork.make_shape(hq, hkv, d, bs, SPORK[dtype], self.scale)
        self.k = torch.full((num_blocks, hkv, bs, d), float("nan"), dtype=dtype, device="cuda")
        self.v = torch.full((num_blocks, hkv, d, bs), float("nan"), dtype=dtype, device="cuda")
        self.table = ints(n, max_blocks)
        self.t = spork.make_tables(bs, self.table, ints(n), ints(num_blocks), ints(num_blocks), ints(2))
        spork.spork_tables_init(self.t, torch.from_numpy(self.rng.permutation(num_blocks).astype(np.int32)).cuda())
        self.tables_ws = torch.empty(spork.spork_tables_workspace_bytes(self.t), dtype=torch.uint8, device="cuda")
        spork.spork_tables_workspace_clear(self.t, self.tables_ws)
        self.chunk_ws = torch.full((spork.spork_chunk_workspace_bytes(self.shape, n, most) // 4,), float("nan"), device="cuda")
        self.lens, self.new, self.parents = ints(n), ints(n), ints(n)
        self.slots = torch.zeros(most, dtype=torch.int64, device="cuda")
        self.positions, self.row_off, self.kv_len = ints(most), ints(n + 1), ints(n)
        self.copies, self.n_copies, self.status = ints(n, 3), ints(1), ints(1)
        self.fused = torch.zeros(most, (hq + 2 * hkv) * d, dtype=dtype, device="cuda")  # q | k | v of a token
        self.k_new = torch.zeros(most, hkv, d, dtype=dtype, device="cuda")
        self.v_new = torch.zeros(most, hkv, d, dtype=dtype, device="cuda")
        self.out = torch.zeros(most, hq, d, dtype=dtype, device="cuda")
        self.lse = torch.zeros(most, hq, dtype=F32, device="cuda")
        self.contexts = [[] for _ in range(n)]

    def launch(self):
        spork.spork_tables_step(self.t, self.lens, self.new, self.parents, self.slots, self.positions, self.row_off, self.kv_len,
                                self.copies, self.n_copies, self.status, self.tables_ws)
        spork.spork_kv_copy_batch(self.shape, self.k, self.v, self.k.shape[0], self.copies, self.n_copies)
        spork.spork_kv_write(self.shape, self.k, self.v, self.k.shape[0], self.slots, self.k_new, self.v_new)
        q = self.fused[:, :self.hq * self.d].unflatten(1, (self.hq, self.d))
        spork.spork_chunk_attn(self.shape, q, self.k, self.v, self.table, self.row_off, self.kv_len, self.out, self.lse, self.chunk_ws)

    def projections(self):
        """New queries, keys and values for `most` tokens."""
        x = torch.from_numpy(self.rng.standard_normal(tuple(self.fused.shape)).astype(np.float32))
        self.fused.copy_(x.to(self.dtype))
        q, k, v = self.fused.split([self.hq * self.d, self.hkv * self.d, self.hkv * self.d], 1)
        self.k_new.copy_(k.unflatten(1, (self.hkv, self.d)))
        self.v_new.copy_(v.unflatten(1, (self.hkv, self.d)))
        self.out.fill_(7.5)
        self.lse.fill_(7.5)

    def tokens(self, lens, new, parents):
        """The step in Python: contexts cut, forked and extended."""
        old, row = self.contexts, 0
        k, v = self.k_new.double().cpu(), self.v_new.double().cpu()
        self.contexts = []
        for s in range(self.n):
            kept = old[parents[s] if parents[s] >= 0 else s][:lens[s]]
            assert len(kept) == lens[s]
            self.contexts.append(kept + [(k[row + i], v[row + i]) for i in range(new[s])])
            row += new[s]

    def check(self, new, tag):
        torch.cuda.synchronize()
        rows = sum(new)
        assert self.status.item() == 0 and self.row_off.tolist() == [0] + np.cumsum(new).tolist()
        assert self.kv_len.tolist() == [len(c) for c in self.contexts]
        held = [(torch.stack([x for x, _ in c]), torch.stack([x for _, x in c])) if c else
                (torch.zeros(0, self.hkv, self.d, dtype=torch.float64),) * 2 for c in self.contexts]
        q = self.fused[:rows, :self.hq * self.d].unflatten(1, (self.hq, self.d)).cpu()
        out, lse, size, mass = attention(q, held, new, self.scale)
        o_tol, l_tol = bounds(self.dtype, out, lse, size, mass, self.scale, max(len(c) for c in self.contexts) + 1, self.d)
        worst_o = ((self.out[:rows].double().cpu() - out).abs() / o_tol).max().item() if rows else 0.0
        worst_l = ((self.lse[:rows].double().cpu() - lse).abs() / l_tol).max().item() if rows else 0.0
        say(f"  {tag}: out at {worst_o:.2f}, lse at {worst_l:.2f} of the bound")
        assert worst_o <= 1 and worst_l <= 1
        assert (self.out[rows:] == 7.5).all() and (self.lse[rows:] == 7.5).all()

    def set(self, lens, new, parents):
        for t, x in ((self.lens, lens), (self.new, new), (self.parents, parents)):
            t.copy_(torch.tensor(x, dtype=torch.int32))


def captured(call):
    """A graph of `call`, which has run once on a side stream before."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


N = -1
STEPS = [  # lens, new tokens, parents of six rows
    ([0] * 6, [200, 37, 0, 0, 0, 0], [N] * 6),                      # prompts, one not yet whole
    ([200, 37, 0, 0, 0, 0], [89, 1, 0, 0, 0, 1], [N] * 6),          # its rest beside single tokens
    ([289, 38, 289, 280, 38, 1], [1, 1, 5, 3, 1, 1], [N, N, 0, 0, 1, N]),   # probes fork, one behind its parent
    ([290, 39, 294, 283, 39, 2], [1, 0, 1, 1, 1, 1], [N] * 6),
    ([285, 39, 290, 283, 32, 0], [6, 1, 1, 0, 1, 0], [N, N, 0, N, N, N]),   # rollbacks, an end, a probe forks again
    ([0, 40, 0, 0, 33, 0], [16, 17, 0, 0, 15, 250], [N] * 6),       # ends, and a new prompt
    ([16, 57, 16, 57, 48, 250], [1, 1, 1, 1, 1, 1], [N, N, 0, 1, N, N]),    # forks at a block's edge and inside one
    ([17, 58, 17, 58, 49, 251], [0] * 6, [N] * 6),                  # nothing new
]


@pytest.mark.parametrize("dtype,hq,hkv,d,bs", [(BF16, 8, 2, 128, 16), (BF16, 4, 4, 64, 32), (F32, 6, 2, 64, 16), (BF16, 5, 1, 128, 32)])
@pytest.mark.parametrize("graph", (False, True))
def test_a_batch_that_forks_rolls_back_and_ends(dtype, hq, hkv, d, bs, graph):
    s = Server(dtype, hq, hkv, d, bs, 6, 80, 24, 300, seed=hq * d + bs)
    call = s.launch
    if graph:
        s.set([0] * 6, [0] * 6, [N] * 6)
        call = captured(s.launch).replay
    for i, (lens, new, parents) in enumerate(STEPS):
        s.projections()
        s.set(lens, new, parents)
        s.tokens(lens, new, parents)
        torch.cuda.synchronize()
        call()
        s.check(new, f"step {i}")


def test_a_refused_step_does_nothing():
    """A step that asks for more blocks than are free, or more tokens than fit: the calls behind it leave pools and
    outputs as they were, and the step that fits comes after it."""
    s = Server(BF16, 4, 2, 64, 16, 3, 20, 16, 300, seed=5)
    steps = [([0, 0, 0], [100, 60, 0], 0), ([100, 60, 0], [20, 1, 200], -2), ([100, 60, 0], [150, 1, 200], -4),
             ([100, 65, 0], [1, 1, 1], -1), ([100, 60, 0], [20, 1, 100], 0)]
    for i, (lens, new, status) in enumerate(steps):
        s.projections()
        s.set(lens, new, [N] * 3)
        before = [x.clone() for x in (s.k, s.v, s.table, s.out, s.lse)]
        s.launch()
        torch.cuda.synchronize()
        assert s.status.item() == status
        if status:
            for x, y in zip((s.k, s.v, s.table, s.out, s.lse), before):
                assert torch.equal(torch.nan_to_num(x.float(), nan=99.0), torch.nan_to_num(y.float(), nan=99.0))
        else:
            s.tokens(lens, new, [N] * 3)
            s.check(new, f"step {i}")


@pytest.mark.parametrize("graph", (False, True))
def test_accepted_drafts_decide_the_next_step(graph):
    """Main rows verify K drafts each step, and what was accepted, known on the GPU alone, is the next step's start."""
    n, k, vocab = 5, 4, 300
    s = Server(BF16, 8, 2, 64, 16, n, 100, 12, n * (k + 1), seed=11)
    logits = torch.zeros(n * (k + 1), vocab, device="cuda")
    drafts = torch.zeros(n, k, dtype=torch.int32, device="cuda")
    accepted, token = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.zeros(spork.spork_verify_workspace_bytes(n, k, vocab), dtype=torch.uint8, device="cuda")

    def step():
        s.launch()
        spork.spork_verify_accept(None, None, None, None, None, None, None, logits, spork.SPORK_DTYPE_F32, vocab, drafts, n, k,
                                  accepted, token, None, ws)
        s.lens.add_(accepted)
        s.lens.add_(1)

    call = step
    if graph:  # (captured over empty rows)
        s.set([0] * n, [0] * n, [N] * n)
        call = captured(step).replay
    first = [1, 3, 5, 2, 4]
    s.projections()
    s.set([0] * n, first, [N] * n)
    s.tokens([0] * n, first, [N] * n)
    s.launch()
    s.check(first, "prompts")
    lens = list(first)
    s.set(lens, [k + 1] * n, [N] * n)
    for i in range(6):
        s.projections()
        s.tokens(lens, [k + 1] * n, [N] * n)
        logits.copy_(torch.from_numpy(s.rng.standard_normal((n * (k + 1), vocab)).astype(np.float32)))
        greedy = logits.argmax(1).view(n, k + 1)
        want = [(i + j) % (k + 1) for j in range(n)]
        drafts.copy_(greedy[:, :k])
        for j, w in enumerate(want):
            if w < k:
                drafts[j, w] = (drafts[j, w] + 1) % vocab
        torch.cuda.synchronize()
        call()
        s.check([k + 1] * n, f"verify {i}")
        assert accepted.tolist() == want and token.tolist() == [greedy[j, w].item() for j, w in enumerate(want)]
        lens = [a + 1 + w for a, w in zip(lens, want)]
        assert s.lens.tolist() == lens


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Launches go to the current device: with another one current, nothing is launched."""
    s = Server(BF16, 4, 2, 64, 16, 2, 9, 4, 8, seed=1)
    s.projections()
    s.set([0, 0], [3, 2], [N] * 2)
    stream = torch.cuda.current_stream()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    q = s.fused[:, :s.hq * s.d].unflatten(1, (s.hq, s.d))
    calls = (lambda: spork.spork_tables_init(s.t, stream=stream),
             lambda: spork.spork_tables_workspace_clear(s.t, s.tables_ws, stream=stream),
             lambda: spork.spork_tables_step(s.t, s.lens, s.new, s.parents, s.slots, s.positions, s.row_off, s.kv_len, s.copies,
                                             s.n_copies, s.status, s.tables_ws, stream=stream),
             lambda: spork.spork_kv_copy_batch(s.shape, s.k, s.v, 9, s.copies, s.n_copies, stream=stream),
             lambda: spork.spork_chunk_attn(s.shape, q, s.k, s.v, s.table, s.row_off, s.kv_len, s.out, s.lse, s.chunk_ws,
                                            stream=stream))
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert (s.out == 7.5).all()


def test_one_row_of_a_wider_buffer():
    """A single query row: the distance to the next one does not matter."""
    s = Server(F32, 4, 2, 64, 16, 1, 9, 4, 1, seed=2)
    s.projections()
    s.set([0], [1], [N])
    s.tokens([0], [1], [N])
    s.launch()
    wide = torch.zeros(1, 4 * 64 + 3, device="cuda")
    wide[:, :256] = s.fused[:, :256]
    spork.spork_chunk_attn(s.shape, wide[:, :256].unflatten(1, (4, 64)), s.k, s.v, s.table, s.row_off, s.kv_len, s.out, s.lse,
                           s.chunk_ws)
    s.check([1], "one row")


def test_two_batches_on_two_streams():
    """Two batches with tables, pools and workspaces of their own, their steps in flight at the same time."""
    servers = [Server(BF16, 8, 2, 128, 16, 6, 80, 24, 300, seed=21), Server(F32, 4, 2, 64, 32, 6, 80, 24, 300, seed=22)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, (lens, new, parents) in enumerate(STEPS):
        for s in servers:
            s.projections()
            s.set(lens, new, parents)
            s.tokens(lens, new, parents)
        torch.cuda.synchronize()
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                s.launch()
        for s in servers:
            s.check(new, f"step {i}")
