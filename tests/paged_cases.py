"""Plain models of the steps whose lengths live on the GPU, shared by their
tests: block tables step by step with Python lists, and attention over paged
contexts in float64, with bounds on how far the kernels may be from it."""
import math

import numpy as np
import torch


def blocks_of(tokens, bs):
    return -(-tokens // bs)


class TablesModel:
    """Rows, references and free queue, changed one queue operation at a time in
    the order that spork.h gives; a step that doesn't fit changes nothing."""

    def __init__(self, n_seqs, num_blocks, bs, max_blocks, order=None):
        self.bs, self.max_blocks, self.num_blocks = bs, max_blocks, num_blocks
        self.rows = [[] for _ in range(n_seqs)]
        self.refs = [0] * num_blocks
        self.queue = list(range(num_blocks)) if order is None else [int(x) for x in order]

    def step(self, lens, new, parents, max_tokens):
        """(status, slots, positions, row_off, kv_len, copies)"""
        n, bs = len(self.rows), self.bs
        parents = [-1] * n if parents is None else list(parents)
        codes = []
        for s in range(n):
            p = parents[s]
            if lens[s] < 0 or new[s] < 0 or p >= n or p == s or (p >= 0 and parents[p] >= 0) or \
                    blocks_of(lens[s], bs) > len(self.rows[p if p >= 0 else s]):
                codes.append(-1)
            elif lens[s] + new[s] > self.max_blocks * bs:
                codes.append(-4)
        if sum(max(x, 0) for x in new) > max_tokens:
            codes.append(-4)
        saved = ([list(r) for r in self.rows], list(self.refs), list(self.queue))
        if not codes:
            try:
                return (0,) + self._run(lens, new, parents)
            except IndexError:  # the queue ran out
                self.rows, self.refs, self.queue = saved
                codes.append(-2)
        return min(codes), [], [], [0] * (n + 1), [0] * n, []

    def _take(self):
        b = self.queue.pop(0)
        self.refs[b] = 1
        return b

    def _run(self, lens, new, parents):
        n, bs = len(self.rows), self.bs
        old = self.rows
        self.rows = [list(old[parents[s] if parents[s] >= 0 else s][:blocks_of(lens[s], bs)]) for s in range(n)]
        for s in range(n):
            if parents[s] >= 0:
                for b in self.rows[s]:
                    self.refs[b] += 1
        for s in range(n):
            for b in old[s][0 if parents[s] >= 0 else blocks_of(lens[s], bs):]:
                self.refs[b] -= 1
                if self.refs[b] == 0:
                    self.queue.append(b)
        slots, positions, off, copies = [], [], [0], []
        for s in range(n):
            row = self.rows[s]
            if new[s] > 0 and lens[s] % bs and self.refs[row[-1]] > 1:
                src = row[-1]
                row[-1] = self._take()
                self.refs[src] -= 1
                copies.append((src, row[-1], lens[s] % bs))
            for i in range(new[s]):
                pos = lens[s] + i
                if pos % bs == 0:
                    row.append(self._take())
                slots.append(row[pos // bs] * bs + pos % bs)
                positions.append(pos)
            off.append(off[-1] + new[s])
        return slots, positions, off, [a + b for a, b in zip(lens, new)], copies


def paged_pools(rng, dtype, hkv, d, bs, kv, spare=3, junk=float("nan"), device="cuda"):
    """Pools with every sequence's context in shuffled blocks and `junk` wherever no token lies; the table, and the
    contexts themselves as float64 [tokens][hkv][d] pairs."""
    held = [blocks_of(k, bs) for k in kv]
    nb = sum(held) + spare
    order = rng.permutation(nb)
    table = np.full((len(kv), max(held + [1])), -7, np.int32)
    kp = torch.full((nb, hkv, bs, d), junk, dtype=torch.float32)
    vp = torch.full((nb, hkv, d, bs), junk, dtype=torch.float32)
    contexts, at = [], 0
    for s, (length, h) in enumerate(zip(kv, held)):
        ids = order[at:at + h]
        at += h
        table[s, :h] = ids
        k = torch.from_numpy(rng.standard_normal((length, hkv, d)).astype(np.float32)).to(dtype)
        v = torch.from_numpy(rng.standard_normal((length, hkv, d)).astype(np.float32)).to(dtype)
        for j, b in enumerate(ids):
            part = slice(j * bs, min((j + 1) * bs, length))
            m = part.stop - part.start
            kp[b, :, :m] = k[part].float().permute(1, 0, 2)
            vp[b, :, :, :m] = v[part].float().permute(1, 2, 0)
        contexts.append((k.double(), v.double()))
    return kp.to(dtype).to(device), vp.to(dtype).to(device), torch.from_numpy(table).to(device), contexts


def attention(q, contexts, new, scale):
    """float64 outputs [rows][hq][d] and lse of the ragged batch, and what the bounds are made of: the outputs over
    |v|, and the largest sum |q||k| of a row's scores."""
    rows, hq, d = q.shape
    out, lse = torch.zeros(rows, hq, d, dtype=torch.float64), torch.full((rows, hq), -math.inf, dtype=torch.float64)
    size, mass = torch.zeros_like(out), torch.zeros(rows, hq, dtype=torch.float64)
    row = 0
    for (k, v), n in zip(contexts, new):
        length, hkv = k.shape[0], k.shape[1]
        if n and length:
            last = length - n + torch.arange(n)
            sees = torch.arange(length)[None] <= last[:, None]
            for h in range(hq):
                kh, vh, qh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)], q[row:row + n, h].double()
                s = (qh @ kh.T) * scale
                s = s.masked_fill(~sees, -math.inf)
                x = torch.logsumexp(s, 1)
                p = torch.where(sees, torch.exp(s - torch.where(x.isinf(), 0.0, x)[:, None]), 0.0)
                out[row:row + n, h], size[row:row + n, h] = p @ vh, p @ vh.abs()
                lse[row:row + n, h] = x
                mass[row:row + n, h] = (qh.abs() @ kh.abs().T).masked_fill(~sees, 0.0).amax(1)
        row += n
    return out, lse, size, mass


def bounds(dtype, out, lse, size, mass, scale, longest, d):
    """How far an output and an lse may be from the float64 ones.

    A score is d products summed in float32 (each product and sum rounded, so at most (d + 2) 2^-24 of sum |q||k|, the
    factor scale * log2 e among them): `off` in the exponent, so probabilities are off by a factor of at most e^(2 off)
    against each other. The exponential (2^-22 with its argument's rounding of up to 2^-24 * |argument|, an argument
    below 150 counting: 150 ln 2 2^-24 < 2^-17) and the sums over `longest` tokens, in float32, in any order, add
    2^-17 + longest 2^-23. bf16 rounds each probability (2^-8) and the output (2^-8); fp32 the output (2^-24)."""
    off = abs(scale) * mass * (d + 4) * 2.0 ** -24
    soft = torch.expm1(2 * off) + 2.0 ** -17 + longest * 2.0 ** -23
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    prob = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    o = size * (soft[..., None] + prob) * (1 + half) + out.abs() * half + 1e-30
    x = torch.where(lse.isinf(), torch.zeros_like(lse), lse)
    return o, off + soft + x.abs() * 2.0 ** -21 + 1e-6
