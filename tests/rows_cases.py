"""Plain models of what happens between a projection's rows and the cache of 8-bit
codes, in float64: norms, rotations, codes and scales, token by token."""
import numpy as np
import torch

LARGEST, LEAST_EXP, MOST_EXP = 448.0, -100, 120


def code_values():
    """What each of the 256 codes stands for, from its bits: sign, four exponent bits (bias 7), three mantissa bits;
    all ones but the sign is no number."""
    out = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        out[c] = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        if c & 127 == 127:
            out[c] = np.nan
        if c & 128:
            out[c] = -out[c]
    return out


VALUES = code_values()
_HELD = VALUES[:127]
_MIDDLE = (_HELD[1:] + _HELD[:-1]) / 2


def encode(x):
    """Nearest codes of |x| <= 448, ties to the even one; what is not finite becomes 127. The sign bit is kept."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    i = np.searchsorted(_MIDDLE, np.where(np.isfinite(a), a, 0))
    tie = (i < 126) & (a == _MIDDLE[np.minimum(i, 125)])
    i = i + (tie & (i % 2 == 1))
    assert (a[np.isfinite(a)] <= LARGEST).all()
    return (np.where(np.isfinite(x), i, 127) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def same_codes(got, want):
    """Equal, but for the sign of what is no number."""
    return ((got == want) | ((got & 127 == 127) & (want & 127 == 127))).all()


def exponent(top):
    """The least allowed e with top <= 448 * 2^e."""
    return next((e for e in range(LEAST_EXP, MOST_EXP) if top <= LARGEST * 2.0 ** e), MOST_EXP)


class PoolModel:
    """The codes (uint8) [blocks][heads][block size][d] and exponents [blocks][heads] of keys, or values."""

    def __init__(self, codes, scale):
        self.codes, self.e = codes.copy(), scale.astype(np.int64) - 127

    def write(self, block, kept, x):
        """Tokens x [n][heads][d] behind the first `kept` of a block."""
        for h in range(self.codes.shape[1]):
            new = x[:, h]
            finite = np.abs(new[np.isfinite(new)])
            e = exponent(finite.max() if finite.size else 0.0)
            if kept:
                old = self.codes[block, h, :kept]
                e = max(e, self.e[block, h])
                if e > self.e[block, h]:
                    self.codes[block, h, :kept] = encode(VALUES[old] * 2.0 ** float(self.e[block, h] - e))
            self.codes[block, h, kept:kept + len(new)] = encode(new * 2.0 ** -float(e))
            self.e[block, h] = e

    def copy(self, src, dst, n):
        self.codes[dst, :, :n], self.e[dst] = self.codes[src, :, :n], self.e[src]

    @property
    def scale(self):
        return (self.e + 127).astype(np.uint8)

    def values(self, block, n):
        """[n][heads][d] of a block's first n tokens."""
        return (VALUES[self.codes[block, :, :n]] * 2.0 ** self.e[block].astype(np.float64)[:, None, None]).swapaxes(0, 1)


def turned(x, weight, eps, positions, inv_freq, magnitude, interleaved):
    """Rows [n][heads][d] in float64: norm (weight None: none) and rotation (inv_freq None: none); and the sizes of what
    the rotation adds up, for bounds."""
    x = np.asarray(x, np.float64).copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    size = np.abs(x)
    if inv_freq is not None:
        half = len(inv_freq)
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        t = np.asarray(positions, np.float64)[:, None, None] * inv_freq
        c, s = magnitude * np.cos(t), magnitude * np.sin(t)
        p, q = x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = p * c - q * s, q * c + p * s
        size[..., a] = size[..., b] = abs(magnitude) * (np.abs(p) + np.abs(q))
    return x, size


def turn_bound(want, size, d, bf16):
    """How far a norm and rotation in float32, rounded once, may be from float64.

    The sum of d squares: each rounded, and d - 1 sums in any order: (d + 1) 2^-24 of it, half of that in its root; the
    mean's and eps' roundings, root and quotient 5 2^-24 more; two products with it. A rotation's cosine and sine are
    rounded (2^-24 each of what they multiply, and the angle in float64 is good to 2^-30), its products and its sum
    likewise: 4 2^-24 of the products' sizes. All of it relative to `size`: (d / 2 + 12) 2^-24, and 2^-28 for the angle.
    Then the output's rounding: 2^-8 in bf16, 2^-24 in float32."""
    off = size * ((d / 2 + 12) * 2.0 ** -24 + 2.0 ** -28)
    return off + (np.abs(want) + off) * (2.0 ** -8 if bf16 else 2.0 ** -24) + 1e-38


def to_f64(t):
    return t.detach().to(torch.float64).cpu().numpy()
