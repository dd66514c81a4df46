"""Where spork_chunk_attn finds its blocks: every query row of the checked tiles is
four times one key of its context, which takes nearly all of the row's softmax, and
the rows' keys lie in every 32-token stage of the context. So a stage that is left
out, read twice in place of another or taken from a block of another place of the
table makes outputs of another token's values, far outside bounds that do not grow
with the context. The shared-stage tiles here walk their table in windows of 64
entries (1,024 or 2,048 positions), three windows or more in a piece.

That such mistakes would show is tested on the CPU, with each of them planted in
the oracle."""
import math

import numpy as np
import pytest
import torch

from gpu_cases import say
from paged_cases import attention, bounds, paged_pools
from paper_2607_03333_amd import spork

BF16, F32 = torch.bfloat16, torch.float32
STAGE = 32


class Needles:
    """One sequence of `rows` new tokens in a context of `length`; `checked` are the query rows that seek a key."""

    def __init__(self, dtype, hq, hkv, d, bs, rows, length, checked, seed=0, device="cuda"):
        rng = np.random.default_rng(seed + hq + d + bs + rows + length)
        self.dtype, self.hq, self.hkv, self.d, self.bs = dtype, hq, hkv, d, bs
        self.rows, self.length, self.checked = rows, length, list(checked)
        self.scale = float(np.float32(1.0 / math.sqrt(d)))
        self.k, self.v, self.table, self.contexts = paged_pools(rng, dtype, hkv, d, bs, [length], device=device)
        keys, group = self.contexts[0][0], hq // hkv
        self.q = torch.from_numpy(rng.standard_normal((rows, hq, d)).astype(np.float32)).to(dtype)
        self.sought = {}
        for i, r in enumerate(self.checked):
            last = length - rows + r
            for h in range(hq):
                p = i * group + h % group  # a KV head's rows take one stage after the other
                t = min(p % (last // STAGE + 1) * STAGE + int(rng.integers(STAGE)), last)
                self.q[r, h] = (4.0 * keys[t, h // group]).to(dtype)
                self.sought[r, h] = t

    def reference(self, contexts=None):
        """Of the checked rows, each the last one of its own context."""
        k, v = contexts or self.contexts[0]
        parts = []
        for r in self.checked:
            end = k.shape[0] - self.rows + r + 1
            parts.append(attention(self.q[r:r + 1].cpu(), [(k[:end], v[:end])], [1], self.scale))
        return [torch.cat(x) for x in zip(*parts)]

    def bounds(self, ref):
        """`longest` of paged_cases.bounds, which counts float32 additions in any order, by the order that the kernel has:
        at most 32 products of a stage in one, then stages, then up to 64 pieces and ways."""
        return bounds(self.dtype, *ref, self.scale, STAGE + self.length // 16 + 64, self.d)

    def run(self):
        rows, dev = self.rows, "cuda"
        shape = spork.make_shape(self.hq, self.hkv, self.d, self.bs, spork.SPORK_DTYPE_BF16 if self.dtype == BF16 else
                                 spork.SPORK_DTYPE_F32, self.scale)
        out = torch.full((rows, self.hq, self.d), 7.5, dtype=self.dtype, device=dev)
        lse = torch.full((rows, self.hq), 7.5, dtype=F32, device=dev)
        ws = torch.full((spork.spork_chunk_workspace_bytes(shape, 1, rows) // 4,), float("nan"), dtype=F32, device=dev)
        spork.spork_chunk_attn(shape, self.q.to(dev), self.k, self.v, self.table, torch.tensor([0, rows], dtype=torch.int32, device=dev),
                               torch.tensor([self.length], dtype=torch.int32, device=dev), out, lse, ws)
        torch.cuda.synchronize()
        return out[self.checked].double().cpu(), lse[self.checked].double().cpu()


def three_tiles(rows, per):
    """The query rows of the first, a middle and the last tile of `per` rows."""
    middle = rows // per // 2 * per
    return [*range(per), *range(middle, middle + per), *range(rows - per, rows)]


@pytest.mark.gpu
@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("dtype,hq,hkv,d,rows,length", [
    (BF16, 64, 8, 128, 1024, 7011),  # 256 tiles of 256 packed rows, about one to a slice: pieces of 6,000 positions
    (BF16, 64, 8, 64, 1024, 7011),
    (BF16, 56, 8, 128, 1100, 7300),  # 252 rows in a tile
    (BF16, 16, 2, 64, 16, 9000),     # four row tiles: stages of each wave's own, two ways
    (BF16, 16, 2, 128, 2, 9000),     # one row tile, eight ways
    (F32, 16, 2, 64, 20, 3000),
    (F32, 16, 2, 128, 2, 3000),
])
def test_every_stage_is_found(dtype, hq, hkv, d, rows, length, bs):
    group = hq // hkv
    per = 256 // group
    c = Needles(dtype, hq, hkv, d, bs, rows, length, three_tiles(rows, per) if rows > 3 * per else range(rows))
    ref = c.reference()
    o_tol, l_tol = c.bounds(ref)
    out, lse = c.run()
    o_off, l_off = (out - ref[0]).abs() / o_tol, (lse - ref[1]).abs() / l_tol
    say(f"  needles: out at {o_off.max().item():.2f}, lse at {l_off.max().item():.2f} of the bound")
    worst = o_off.amax((1, 2)).argmax().item()
    assert (o_off <= 1).all(), f"row {c.checked[worst]}: {[c.sought[c.checked[worst], h] for h in range(hq)]}"
    assert (l_off <= 1).all()


def faults(length, window):
    """Positions in the order in which a mistaken walk reads them, by the mistake."""
    at = np.arange(length)
    yield "a window read twice, the next one not", np.where(at // window == 2, at - window, at)
    yield "windows that lag from the second on", np.where(at >= window, at - window, at)
    yield "a window left out", at[at // window != 1]
    yield "the last window left out", at[at // window != (length - 1) // window]
    middle = length // STAGE // 2
    yield "a stage left out", at[at // STAGE != middle]
    yield "a stage read twice, the next one not", np.where(at // STAGE == middle, at - STAGE, at)
    yield "two blocks exchanged for others", np.where(at // 16 % 64 == 63, at - 48, at)


@pytest.mark.parametrize("d,bs", [(64, 16), (128, 16), (64, 32), (128, 32)])
def test_mistaken_walks_would_show(d, bs):
    """One KV head's tile of 256 packed rows: each mistake puts an output of the oracle out of its bound."""
    c = Needles(BF16, 8, 1, d, bs, 32, 7011, range(32), device="cpu")
    ref = c.reference()
    o_tol, _ = c.bounds(ref)
    k, v = c.contexts[0]
    weight = torch.exp(4.0 * c.scale * (k[list(c.sought.values()), 0] ** 2).sum(1) - ref[1].flatten())
    assert weight.median() > 0.99  # of the key that a row seeks
    for what, order in faults(c.length, 64 * bs):
        order = torch.from_numpy(order)
        off = (c.reference((k[order], v[order]))[0] - ref[0]).abs() / o_tol
        assert off.max() > 10, what
