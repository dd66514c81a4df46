"""Attention over the cache of 8-bit codes in batches of so many sequences that a
tile takes several KV heads (spork_kvq_attn), for sequences of one to eight row tiles
of 32 packed rows and of several tiles, side by side, against the definition in
float64: outputs and lse."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import BF16, F32
from test_gpu_kvq_attn import Case

pytestmark = pytest.mark.gpu

# Packed rows (rows times query heads of a KV head) of a sequence: each number of row tiles, at both of its ends.
PACKED = (1, 32, 33, 64, 65, 80, 96, 97, 112, 128, 129, 160, 192, 224, 256, 257)

# hq, hkv, sequences: 512, 768, 1,024 and 2,048 tiles and a few more, of two, four and eight KV heads where there are
# rows for that; the numbers of KV heads that these do not divide too.
BATCHES = [(32, 4, 128), (32, 4, 192), (64, 8, 128), (32, 8, 256), (16, 16, 64), (18, 6, 172), (21, 3, 171), (12, 12, 171)]


def batch(hq, hkv, n, seed):
    """New tokens and context lengths of n sequences: the sizes of PACKED in turn between single tokens, contexts of nothing
    else, of some stages, and a few that slices cut."""
    rng = np.random.default_rng(seed)
    group = hq // hkv
    new = [1 if i % 3 == 2 else max(1, PACKED[i % len(PACKED)] // group) for i in range(n)]
    kv = [r + (0, int(rng.integers(1, 40)), int(rng.integers(100, 300)))[i % 3] for i, r in enumerate(new)]
    for i in range(0, n, 37):
        kv[i] += 900
    return new, kv


@pytest.mark.parametrize("bs", (16, 32))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("hq,hkv,n", BATCHES)
def test_tiles_of_several_heads_beside_tiles_of_many_rows(hq, hkv, n, d, bs):
    new, kv = batch(hq, hkv, n, d + bs)
    Case(BF16, hq, hkv, d, bs, new, kv, gain=2.0).run_and_check(f"{n} sequences, {hq}/{hkv} heads")


@pytest.mark.parametrize("packed", (64, 65, 96, 97, 128, 129))
@pytest.mark.parametrize("hq,hkv,n", [(16, 4, 128), (8, 8, 128)])
def test_sequences_of_the_same_number_of_rows(hq, hkv, n, packed):
    """No sequence is another's neighbour of more or fewer row tiles: contexts differ alone."""
    rows = -(-packed // (hq // hkv))
    rng = np.random.default_rng(packed)
    Case(BF16, hq, hkv, 64, 16, [rows] * n, [rows + int(x) for x in rng.integers(0, 200, n)]).run_and_check(f"{packed} packed rows")


@pytest.mark.parametrize("lse", (False, True))
def test_forked_threads_that_verify(lse):
    """64 threads with nine rows each, eight drafts behind their last token, among 192; 32 query and 4 KV heads."""
    rng = np.random.default_rng(1)
    new = [9 if i % 3 == 0 else 1 for i in range(192)]
    c = Case(BF16, 32, 4, 128, 16, new, [r + int(x) for r, x in zip(new, rng.integers(1, 700, 192))])
    c.run(lse=lse)
    if not lse:
        assert (c.lse == 7.5).all()
        want = c.out.clone()
        c.out.fill_(7.5)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(want, c.out)
    c.check("verify")


@pytest.mark.parametrize("n", (128, 192))
def test_openers_of_forks(n):
    """Forks' first rows, 8 to 50 of them."""
    rng = np.random.default_rng(2)
    new = [int(x) for x in rng.integers(8, 51, n)]
    Case(BF16, 32, 4, 128, 16, new, [r + int(x) for r, x in zip(new, rng.integers(0, 300, n))]).run_and_check("openers")


@pytest.mark.parametrize("hq,hkv,n,d", [(16, 4, 128, 64), (8, 8, 256, 64), (6, 6, 171, 128)])
def test_fp32_tiles_of_several_heads(hq, hkv, n, d):
    new, kv = batch(hq, hkv, n, d)
    Case(F32, hq, hkv, d, 16, new, kv).run_and_check("fp32")
