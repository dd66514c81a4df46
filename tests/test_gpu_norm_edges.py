"""Norms of queries and keys (spork_qk_rope) and of the queries of a write
(spork_kvq_write) where a factor leaves the range of 32 bits and the result doesn't,
against the definition in float64: heads of zeros under the smallest eps, the
largest eps that is taken, weights that undo the factor. The bound is that of every norm
(rows_cases.turn_bound), and for channels that the norm takes below 2^-126 what 32 bits
hold of them: a channel over its head's root is a multiple of 2^-149 there, half of that
off, and is then multiplied by its weight; a rotation adds two such."""
import numpy as np
import pytest
import torch

from gpu_cases import say
from paper_2607_03333_amd import spork
from rows_cases import to_f64, turn_bound, turned
from test_gpu_rope import BF16, F32, SPORK

pytestmark = pytest.mark.gpu

HQ, HKV, N = 4, 2, 5


def normed(dtype, d, gain, weight, eps, rotary, write, zeros=()):
    """Rows of sizes about `gain` (those of `zeros` all zero), normed with weights about `weight`; compared head by head."""
    rng = np.random.default_rng(d + rotary)
    x = torch.from_numpy(rng.standard_normal((N, HQ + 2 * HKV, d)) * gain).to(dtype).cuda()
    for row in zeros:
        x[row] = 0
    q, k, v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
    weights = [torch.from_numpy(rng.uniform(0.5, 1.5, d) * weight).to(dtype).cuda() for _ in range(2)]
    inv_freq = spork.spork_rope_frequencies(rotary, 1e4)[0] if rotary else None
    pos = np.arange(3, 3 + N, dtype=np.int32)
    shape = spork.make_shape(HQ, HKV, d, 16, SPORK[dtype], 1.0)
    rope = spork.make_rope(torch.from_numpy(inv_freq).cuda()) if rotary else None
    norm = spork.make_qk_norm(*weights, eps)
    positions = torch.from_numpy(pos).cuda()
    q_out, k_out = (torch.full((N, h, d), 7.5, dtype=dtype, device="cuda") for h in (HQ, HKV))
    pairs = [(q, weights[0], q_out)]
    if write:
        u8 = lambda *m: torch.zeros(m, dtype=torch.uint8, device="cuda")  # noqa: E731
        cache = spork.make_kvq(u8(1, HKV, 16, d), u8(1, HKV, d, 16), u8(1, HKV), u8(1, HKV))
        spork.spork_kvq_write(shape, cache, rope, norm, positions.long(), positions if rope else None, q, k, v, q_out)
    else:
        spork.spork_qk_rope(shape, rope, norm, positions if rope else None, q, k, q_out, k_out)
        pairs.append((k, weights[1], k_out))
    torch.cuda.synchronize()
    for x, w, got in pairs:
        want, size = turned(to_f64(x), to_f64(w), eps, pos, inv_freq, 1.0, False)
        assert np.isfinite(want).all() and np.abs(want).max() < 1e38
        least = 2.0 ** -149 * np.abs(to_f64(w)).max()
        off = np.abs(to_f64(got) - want) / (turn_bound(want, size, d, dtype == BF16) + least)
        assert (off <= 1).all(), f"off by {np.nanmax(off):.3g} of the bound"
        say(f"  norm of {gain:g} by {weight:g}, eps {eps:g}: at {off.max():.2f} of the bound")


BOTH = [pytest.mark.parametrize("write", (False, True)), pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])]


def both(test):
    for mark in BOTH:
        test = mark(test)
    return test


@both
@pytest.mark.parametrize("rotary", (0, 32))
@pytest.mark.parametrize("eps", (5e-324, 1e-300, 1e-150, 1e-77, 1e-60, 1e-38, 1e-27, 1e-26, 1e-6, 1e30))
def test_heads_of_zeros(dtype, d, write, eps, rotary):
    """Zero over the root of any eps is zero, whether 32 bits hold that root or not."""
    normed(dtype, d, 1.0, 1.0, eps, rotary, write, zeros=(0, 3))


@both
@pytest.mark.parametrize("gain,weight,eps", [(1.0, 1.0, 2.0 ** 100), (1e20, 1.0, 1e30), (1.0, 1e30, 1e30), (1e-30, 1e37, 1e30),
                                             (1e-30, 1e37, 1e10), (1e37, 1.0, 1e30), (1e18, 1.0, 1e30), (1e-20, 1.0, 1e-26),
                                             (1e-20, 1.0, 1e-27), (1e-13, 1e20, 1e-26), (1e-38, 1e10, 1e-27)])
def test_eps_of_any_size(dtype, d, write, gain, weight, eps):
    normed(dtype, d, gain, weight, eps, 32, write)


@both
@pytest.mark.parametrize("gain,weight", [(1e-12, 1e32), (1e-10, 1e36), (1e-30, 1e36), (1e17, 1e-30), (1e17, 1e-25), (1e30, 1e-30),
                                         (1e-12, 1e-20), (1e17, 1e20)])
def test_weights_that_undo_the_factor(dtype, d, write, gain, weight):
    normed(dtype, d, gain, weight, 0.0, 32, write)
