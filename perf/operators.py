"""The serving step whose lengths live on the GPU, as cases that can be timed.

Two operators: the block tables and slots of a step built on the GPU from
request lengths (``spork_tables_step``, with the copies of its copy-on-write by
``spork_kv_copy_batch``), and the attention of its new tokens, prompt chunks and
single tokens alike, over the paged cache (``spork_chunk_attn``).

``own`` chooses between the library's calls and the same in plain torch.
``listed()`` are sizes that a server meets, ``draw(rng)`` spreads them over
their ranges. Lengths come from the case itself (``lens``), values from the seed.
"""

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_ELEM = {"bf16": 2, "f32": 4}

# Query heads, KV heads and head size: the models that the library's workloads are shaped on, and other groupings.
QWEN3_4B = dict(hq=32, hkv=8, d=128)
QWEN3_32B = dict(hq=64, hkv=8, d=128)
QWEN3_30B_A3B = dict(hq=32, hkv=4, d=128)
SMALL_F32 = dict(hq=4, hkv=2, d=64)
GROUPS_OF_7 = dict(hq=28, hkv=4, d=128)
NARROW_HEADS = dict(hq=16, hkv=16, d=64)
ONE_KV_HEAD = dict(hq=16, hkv=1, d=128)


def _chunk(name, heads, **kw):
    """An attention call: `chunks` sequences with chunk_lo..chunk_hi new tokens and `singles` with one, each behind
    ctx_lo..ctx_hi tokens of context. `fused`: the query rows lie inside rows that hold keys and values too."""
    case = dict(name=name, kind="chunk", dtype="bf16", block_size=16, chunks=0, chunk_lo=1, chunk_hi=1, singles=0,
                ctx_lo=0, ctx_hi=0, fused=False, q_gain=1.0, lens=1)
    case.update(heads)
    case.update(kw)
    return case


def _tables(name, **kw):
    """A tables step: `sessions` main rows of len_lo..len_hi tokens, rolled back by up to `back` tokens (rejected drafts),
    that append new_lo..new_hi; `probes` rows of each fork there and append open_lo..open_hi. hkv > 0: the
    copy-on-write of the pools (bf16) follows."""
    case = dict(name=name, kind="tables", block_size=16, sessions=1, probes=0, len_lo=1, len_hi=1, back=0, new_lo=1,
                new_hi=1, open_lo=0, open_hi=0, hkv=0, d=128, lens=1)
    case.update(kw)
    return case


def listed():
    return [
        # One user's next token behind a short context: the latency of the launches.
        _chunk("one-token", QWEN3_4B, singles=1, ctx_lo=1000, ctx_hi=1000),
        # A decode batch of very different lengths, the queries inside the rows of a fused projection.
        _chunk("decode-ragged", QWEN3_4B, singles=96, ctx_lo=3, ctx_hi=8190, fused=True, q_gain=3.0),
        # Two very long contexts, one token each: few rows, a long axis.
        _chunk("decode-long", QWEN3_30B_A3B, singles=2, ctx_lo=120000, ctx_hi=131070, block_size=32),
        # The whole of a prompt in one chunk.
        _chunk("whole-prompt", QWEN3_4B, chunks=1, chunk_lo=4096, chunk_hi=4096),
        # A late chunk of a long prompt: the largest.
        _chunk("late-chunk", QWEN3_32B, chunks=1, chunk_lo=2048, chunk_hi=2048, ctx_lo=30000, ctx_hi=30000, q_gain=3.0),
        # Chunks of prompts beside sequences that decode, as a server mixes them.
        _chunk("chunks-and-tokens", QWEN3_30B_A3B, chunks=3, chunk_lo=300, chunk_hi=512, singles=29, ctx_lo=1, ctx_hi=8000),
        # Short prompts of odd lengths, narrow heads without grouping, 32-token blocks.
        _chunk("short-prompts", NARROW_HEADS, chunks=24, chunk_lo=1, chunk_hi=777, block_size=32, fused=True),
        # The full-precision path.
        _chunk("chunks-f32", SMALL_F32, dtype="f32", chunks=3, chunk_lo=50, chunk_hi=200, singles=2, ctx_lo=0, ctx_hi=900),
        # One session: a probe forks inside a block and both append, with the copy of the shared block.
        _tables("fork-one", sessions=1, probes=1, len_lo=250, len_hi=250, new_lo=1, new_hi=1, open_lo=8, open_hi=8, hkv=2,
                d=64),
        # A decode step of a large batch.
        _tables("tables-decode", sessions=256, len_lo=1, len_hi=8191),
        # Sixteen prompts arrive, the tables of 65 thousand tokens.
        _tables("tables-prompts", sessions=16, len_lo=0, len_hi=0, new_lo=4000, new_hi=4096),
        # After a verify step: mains lose their rejected drafts, two probes of each fork with their openers, blocks are copied.
        _tables("fork-and-verify", sessions=64, probes=2, len_lo=500, len_hi=32768, back=8, new_lo=9, new_hi=9, open_lo=8,
                open_hi=50, hkv=4),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1))))))


# Most that a drawn case may cost: by type, bytes and operations below those of the largest listed case.
_MOST = {"bf16": (9e8, 2.0e12), "f32": (2e8, 2e10)}
_MOST_SCORES = 4.2e9  # padded score elements of the plain form


def draw(rng):
    if rng.random() < 0.3:
        fork = rng.random() < 0.6
        case = _tables("", block_size=rng.choice((16, 16, 32)), sessions=_log_int(rng, 1, 64 if fork else 512),
                       len_hi=_log_int(rng, 2, 16384), lens=rng.randrange(1 << 20))
        case["len_lo"] = rng.choice((0, 1 + case["len_hi"] // 2))
        case["new_hi"] = _log_int(rng, 1, max(1, min(2048, 65536 // case["sessions"])))
        case["new_lo"] = rng.choice((0, case["new_hi"], 1 + case["new_hi"] // 2))
        case["back"] = rng.choice((0, 8, 50))
        if fork:
            open_hi = _log_int(rng, 1, 50)
            case.update(probes=rng.randint(1, 4), open_hi=open_hi, open_lo=rng.choice((0, open_hi)),
                        hkv=rng.choice((0, 2, 4, 8)), d=rng.choice((64, 128)))
        del case["name"]
        return case
    while True:
        f32 = rng.random() < 0.15
        heads = dict(SMALL_F32, d=rng.choice((64, 128))) if f32 else rng.choice(
            (QWEN3_4B, QWEN3_32B, QWEN3_30B_A3B, GROUPS_OF_7, NARROW_HEADS, ONE_KV_HEAD))
        mode = rng.choice(("singles", "chunks", "both"))
        ctx_hi = _log_int(rng, 1, 2048 if f32 else 32768)
        chunk_hi = _log_int(rng, 2, 256 if f32 else 4096)
        case = _chunk("", heads, dtype="f32" if f32 else "bf16", block_size=rng.choice((16, 16, 32)),
                      chunks=0 if mode == "singles" else _log_int(rng, 1, 16),
                      singles=0 if mode == "chunks" else _log_int(rng, 1, 128), chunk_hi=chunk_hi,
                      chunk_lo=rng.choice((1, chunk_hi, 1 + chunk_hi // 2)), ctx_hi=ctx_hi,
                      ctx_lo=rng.choice((0, ctx_hi, 1 + ctx_hi // 2)), fused=rng.random() < 0.4,
                      q_gain=rng.choice((1.0, 3.0)), lens=rng.randrange(1 << 20))
        del case["name"]
        new, kv = _lengths(case)
        w, most = work(case), _MOST[case["dtype"]]
        scores = len(new) * max(new) * case["hq"] * max(kv)
        cache = len(new) * max(kv) * case["hkv"] * case["d"]
        if w["bytes"] <= most[0] and w["flops"] <= most[1] and scores <= _MOST_SCORES and cache <= 2e9:
            return case


# ---- what a case's lengths are ---------------------------------------------------------
def _lengths(case):
    """New tokens and context length with them of every sequence of an attention case; the single tokens are spread among
    the chunks."""
    r = random.Random(case["lens"])
    new = [r.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["chunks"])] + [1] * case["singles"]
    r.shuffle(new)
    return new, [n + r.randint(case["ctx_lo"], case["ctx_hi"]) for n in new]


def _rows(case):
    """(parent, tokens before, tokens held, new tokens) of every table row: a session's main row, then its probes'."""
    r = random.Random(case["lens"])
    out = []
    for _ in range(case["sessions"]):
        main, n = len(out), r.randint(case["len_lo"], case["len_hi"])
        out.append((-1, n, n + r.randint(0, case["back"]), r.randint(case["new_lo"], case["new_hi"])))
        out += [(main, n, 0, r.randint(case["open_lo"], case["open_hi"])) for _ in range(case["probes"])]
    return out


def _blocks(n, bs):
    return (n + bs - 1) // bs


def work(case):
    if case["kind"] == "chunk":
        new, kv = _lengths(case)
        hq, hkv, d, e = case["hq"], case["hkv"], case["d"], _ELEM[case["dtype"]]
        # row r of n sees kv - n + 1 + r positions
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, kv))
        rows = sum(new)
        tables = 4 * sum(_blocks(k, case["block_size"]) for k in kv) + 8 * len(new)
        return {"bytes": rows * hq * (2 * d * e + 4) + 2 * sum(kv) * hkv * d * e + tables, "flops": 4 * hq * d * pairs}
    bs, rows = case["block_size"], _rows(case)
    tokens = sum(r[3] for r in rows)
    taken = sum(_blocks(r[1] + r[3], bs) - _blocks(r[1], bs) for r in rows)
    forked = sum(_blocks(r[1], bs) for r in rows if r[0] >= 0)
    moved = 0
    if case["hkv"]:  # all but one of a session's rows that append inside a shared block copy it
        for s in range(0, len(rows), case["probes"] + 1):
            group = [r for r in rows[s:s + case["probes"] + 1] if r[3] > 0 and r[1] % bs]
            copies = min(len(group), case["probes"])
            moved += copies * (rows[s][1] % bs) * case["hkv"] * case["d"] * 2 * 2 * 2
    # a row's length, new tokens, parent and blocks held in, the last, its offset and its context out; a new token's slot
    # and position; a taken block's queue entry, table entry and references; a forked block's entry twice and references
    return {"bytes": 28 * len(rows) + 12 * tokens + 12 * taken + 16 * forked + moved, "flops": 0}


# ---- inputs ----------------------------------------------------------------------------
def _gen(seed, part):
    return torch.Generator(device=DEVICE).manual_seed(seed * 16 + part)


def _normal(shape, dtype, gen, gain=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32) * gain).to(_TORCH[dtype])


def _ints(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype).to(DEVICE)


def _prepare_chunk(case, seed):
    new, kv = _lengths(case)
    hq, hkv, d, bs, dtype = case["hq"], case["hkv"], case["d"], case["block_size"], case["dtype"]
    n, rows, held = len(new), sum(new), [_blocks(k, bs) for k in kv]
    blocks, most = sum(held) + 8, max(held)
    order = np.random.default_rng(seed).permutation(blocks)
    table = np.zeros((n, most), np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    width = (hq + 2 * hkv) * d if case["fused"] else hq * d
    q = _normal((rows, width), dtype, _gen(seed, 1), case["q_gain"])[:, :hq * d].unflatten(1, (hq, d))
    return dict(kind="chunk", heads=(hq, hkv, d, bs), dtype=dtype, scale=float(np.float32(1.0 / math.sqrt(d))), q=q,
                k_pool=_normal((blocks, hkv, bs, d), dtype, _gen(seed, 2)),
                v_pool=_normal((blocks, hkv, d, bs), dtype, _gen(seed, 3)), blocks=blocks, table=_ints(table),
                row_off=_ints(np.cumsum([0] + new)), kv_len=_ints(kv), most_new=max(new), most_kv=max(kv),
                out=torch.zeros((rows, hq, d), dtype=_TORCH[dtype], device=DEVICE),
                lse=torch.zeros((rows, hq), dtype=torch.float32, device=DEVICE), workspace={})


def _prepare_tables(case, seed):
    bs, rows = case["block_size"], _rows(case)
    n, tokens = len(rows), sum(r[3] for r in rows)
    held = np.array([_blocks(r[2], bs) for r in rows], np.int32)
    most = max(1, max(_blocks(max(r[2], r[1] + r[3]), bs) for r in rows))
    blocks = int(held.sum()) + sum(_blocks(r[1] + r[3], bs) - r[1] // bs + 1 for r in rows) + 8
    order = np.random.default_rng(seed).permutation(blocks).astype(np.int32)
    table = np.zeros((n, most), np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    refs = np.zeros(blocks, np.int32)
    refs[order[:at]] = 1
    queue = np.concatenate([order[at:], np.zeros(at, np.int32)])
    zeros = lambda *m, t=torch.int32: torch.zeros(m, dtype=t, device=DEVICE)  # noqa: E731
    st = dict(kind="tables", n=n, most=most, blocks=blocks, bs=bs, tokens=tokens, table=_ints(table), held=_ints(held),
              refcount=_ints(refs), free_queue=_ints(queue), queue=_ints([0, blocks - at]), lens=_ints([r[1] for r in rows]),
              new=_ints([r[3] for r in rows]), parents=_ints([r[0] for r in rows]) if case["probes"] else None,
              slots=zeros(tokens, t=torch.int64), positions=zeros(tokens), row_off=zeros(n + 1), kv_len=zeros(n),
              copies=zeros(n, 3), n_copies=zeros(1), status=zeros(1), workspace={}, k_pool=None, v_pool=None)
    if case["hkv"]:  # one block more than the tables know, where the plain form puts what is no copy
        hkv, d = case["hkv"], case["d"]
        st.update(heads=(hkv, hkv, d, bs),
                  k_pool=_normal((blocks + 1, hkv, bs, d), "bf16", _gen(seed, 2)),
                  v_pool=_normal((blocks + 1, hkv, d, bs), "bf16", _gen(seed, 3)))
    return st


def prepare(case, seed):
    return _prepare_chunk(case, seed) if case["kind"] == "chunk" else _prepare_tables(case, seed)


# ---- one pass --------------------------------------------------------------------------
def _chunk_own(s):
    from paper_2607_03333_amd import spork
    ws = s["workspace"]
    if not ws:  # made once, as a server does
        ws["shape"] = spork.make_shape(*s["heads"], spork.SPORK_DTYPE_BF16 if s["dtype"] == "bf16" else
                                       spork.SPORK_DTYPE_F32, s["scale"])
        need = spork.spork_chunk_workspace_bytes(ws["shape"], len(s["kv_len"]), len(s["q"]))
        ws["chunk"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)
    spork.spork_chunk_attn(ws["shape"], s["q"], s["k_pool"], s["v_pool"], s["table"], s["row_off"], s["kv_len"], s["out"],
                           s["lse"], ws["chunk"])
    return {k: s[k] for k in ("out", "lse")}


def _tables_own(s):
    from paper_2607_03333_amd import spork
    ws = s["workspace"]
    if not ws:
        ws["tables"] = spork.make_tables(s["bs"], s["table"], s["held"], s["refcount"], s["free_queue"], s["queue"])
        need = spork.spork_tables_workspace_bytes(ws["tables"])
        ws["scratch"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEVICE)
        spork.spork_tables_workspace_clear(ws["tables"], ws["scratch"])
        if s["k_pool"] is not None:
            ws["shape"] = spork.make_shape(*s["heads"], spork.SPORK_DTYPE_BF16, 1.0)
    spork.spork_tables_step(ws["tables"], s["lens"], s["new"], s["parents"], s["slots"], s["positions"], s["row_off"],
                            s["kv_len"], s["copies"], s["n_copies"], s["status"], ws["scratch"])
    if s["k_pool"] is not None:
        spork.spork_kv_copy_batch(ws["shape"], s["k_pool"], s["v_pool"], s["blocks"], s["copies"], s["n_copies"])


def _chunk_plain(s):
    """The padded batch: every sequence's context gathered from its blocks, all its rows against all of it."""
    q, table, kv_len, off = s["q"], s["table"].long(), s["kv_len"].long(), s["row_off"].long()
    rows, hq, d = q.shape
    n, hkv, most_new, most_kv = len(kv_len), s["k_pool"].shape[1], s["most_new"], s["most_kv"]
    g = hq // hkv
    bs = s["k_pool"].shape[2]
    tokens = table.shape[1] * bs
    k = s["k_pool"][table].float().permute(0, 2, 1, 3, 4).reshape(n, hkv, tokens, d)[:, :, :most_kv]
    v = s["v_pool"][table].float().permute(0, 2, 1, 4, 3).reshape(n, hkv, tokens, d)[:, :, :most_kv]
    at = torch.arange(most_kv, device=DEVICE)
    v = torch.where(at[None, None, :, None] < kv_len[:, None, None, None], v, 0.0)
    j = torch.arange(most_new, device=DEVICE)
    new = off[1:] - off[:-1]
    pick = torch.clamp(off[:-1, None] + j, max=rows - 1)
    qp = q[pick].float().reshape(n, most_new, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most_new * g, d)
    scores = torch.matmul(qp, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    sees = at[None, None] <= (kv_len - new)[:, None, None] + j[None, :, None]  # [n, new, kv]
    scores = scores.reshape(n, hkv, most_new, g, most_kv).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n, hkv, most_new * g, most_kv), v.contiguous()).reshape(n, hkv, most_new, g, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(n, most_new, hq, d)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(n, most_new, hq)
    r = torch.arange(rows, device=DEVICE)
    seq = torch.searchsorted(off[1:].contiguous(), r, right=True)
    return {"out": o[seq, r - off[seq]].to(q.dtype), "lse": lse[seq, r - off[seq]].contiguous()}


def _aside(ids, wanted, size):
    """The wanted places' ids, flat, the others spread behind the last of `size` ids."""
    flat = ids.reshape(-1)
    return torch.where(wanted.reshape(-1), flat, size + torch.arange(flat.numel(), device=DEVICE) % 4096)


def _count(to, size):
    """How often each of the ids occurs."""
    return torch.zeros(size + 4096, dtype=torch.int64, device=DEVICE).index_add_(0, to, torch.ones_like(to))[:size]


def _last(to, size):
    """The last place that holds each of the ids, -1 for none."""
    order = torch.arange(to.numel(), device=DEVICE)
    return torch.full((size + 4096,), -1, device=DEVICE).scatter_reduce_(0, to, order, "amax")[:size]


def _tables_plain(s):
    bs, blocks, n, most = s["bs"], s["blocks"], s["n"], s["most"]
    lens, new, held, table = s["lens"].long(), s["new"].long(), s["held"].long(), s["table"].long()
    row, col = torch.arange(n, device=DEVICE), torch.arange(most, device=DEVICE)[None]
    keep = (lens + bs - 1) // bs
    refs, start, count = s["refcount"].long(), s["queue"][0].long(), s["queue"][1].long()
    parents = torch.full_like(lens, -1) if s["parents"] is None else s["parents"].long()
    forked = parents >= 0
    # forks: the parent's first blocks, one reference more for each
    gets = forked[:, None] & (col < keep[:, None])
    source = table[torch.where(forked, parents, row)]
    refs = refs + _count(_aside(source, gets, blocks), blocks)
    # releases in row and table order: the one that leaves a block without references puts it at the queue's back
    gives = (col >= torch.where(forked, 0, keep)[:, None]) & (col < held[:, None])
    ids, given = table.reshape(-1), _aside(table, gives, blocks)
    refs = refs - _count(given, blocks)
    frees = gives.reshape(-1) & (_last(given, blocks)[ids] == torch.arange(n * most, device=DEVICE)) & (refs[ids] == 0)
    place = _aside((start + count + frees.cumsum(0) - 1) % blocks, frees, blocks)
    ring = torch.cat([s["free_queue"].long(), refs.new_zeros(4096)]).scatter_(0, place, ids)[:blocks]
    count = count + frees.sum()
    table = torch.where(gets, source, table)
    # appends: a copy of the last block where others hold it (the last holder writes in place), then the new blocks
    inside = (lens % bs != 0) & (new > 0)
    tail_col = torch.clamp(lens // bs, max=most - 1)
    tail = table.gather(1, tail_col[:, None])[:, 0]
    tails = _aside(tail, inside, blocks)
    copies = inside & (refs[tail] > 1) & ~((_count(tails, blocks)[tail] == refs[tail]) & (_last(tails, blocks)[tail] == row))
    grow = (lens + new + bs - 1) // bs - keep
    takes = copies + grow
    first = takes.cumsum(0) - takes
    is_copy = copies[:, None] & (col == tail_col[:, None])
    fresh = is_copy | ((col >= keep[:, None]) & (col < (keep + grow)[:, None]))
    nth = first[:, None] + torch.where(is_copy, 0, copies[:, None] + col - keep[:, None])
    table = torch.where(fresh, ring[(start + nth) % blocks], table)
    refs = refs - _count(_aside(tail, copies, blocks), blocks)
    refs = torch.cat([refs, refs.new_zeros(4096)]).index_fill_(0, _aside(table, fresh, blocks), 1)[:blocks]
    taken = takes.sum()
    # the copies in row order, the offsets, and every new token's place
    to = torch.where(copies, copies.cumsum(0) - 1, n)
    listed_ = torch.cat([s["copies"].long(), refs.new_zeros(1, 3)])
    listed_[to] = torch.stack([tail, table.gather(1, tail_col[:, None])[:, 0], lens % bs], 1)
    off = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(s["tokens"], device=DEVICE)
    seq = torch.searchsorted(off[1:].contiguous(), t, right=True)
    pos = lens[seq] + t - off[seq]
    short = taken > count
    for name, value in dict(table=table, held=keep + grow, refcount=refs, free_queue=ring, kv_len=lens + new, row_off=off,
                            queue=torch.stack([(start + taken) % blocks, count - taken]), copies=listed_[:-1],
                            n_copies=copies.sum()[None], status=torch.where(short, -2, 0)[None],
                            slots=table[seq, pos // bs] * bs + pos % bs, positions=pos).items():
        s[name].copy_(value)
    if s["k_pool"] is None:
        return
    c = s["copies"].long()
    real = (row < s["n_copies"])
    src, dst = (torch.where(real, c[:, i], blocks) for i in (0, 1))
    part = torch.arange(bs, device=DEVICE)[None] < torch.where(real, c[:, 2], 0)[:, None]
    k, v = s["k_pool"], s["v_pool"]
    k[dst] = torch.where(part[:, None, :, None], k[src], k[dst])
    v[dst] = torch.where(part[:, None, None, :], v[src], v[dst])


def run(s):
    if s["kind"] == "chunk":
        return _chunk_own(s) if own else _chunk_plain(s)
    if own:
        _tables_own(s)
    else:
        _tables_plain(s)
    names = ("table", "held", "refcount", "free_queue", "queue", "slots", "positions", "row_off", "kv_len", "copies",
             "n_copies", "status") + (() if s["k_pool"] is None else ("k_pool", "v_pool"))
    return {k: s[k] for k in names}


# ---- the attention in 64 bits ------------------------------------------------------------
def exact(case, seed):
    """Sequence by sequence and head by head, from the definition; nothing of a tables step is a computed number."""
    if case["kind"] != "chunk":
        return None
    s = _prepare_chunk(case, seed)
    new, kv = _lengths(case)
    group = case["hq"] // case["hkv"]
    scale = s["scale"]
    out, lse = s["out"].double(), s["lse"].double()
    row = 0
    for i, (m, length) in enumerate(zip(new, kv)):
        ids = s["table"][i, :_blocks(length, case["block_size"])].long()
        last = length - m + torch.arange(m, device=DEVICE)
        hidden = torch.arange(length, device=DEVICE)[None] > last[:, None]
        for h in range(case["hkv"]):
            keys = s["k_pool"][ids, h].reshape(-1, case["d"])[:length].double()
            values = s["v_pool"][ids, h].transpose(1, 2).reshape(-1, case["d"])[:length].double()
            for head in range(h * group, (h + 1) * group):
                x = (s["q"][row:row + m, head].double() @ keys.t().contiguous()).mul_(scale)
                x.masked_fill_(hidden, -math.inf)
                lse[row:row + m, head] = torch.logsumexp(x, 1)
                out[row:row + m, head] = torch.softmax(x, 1) @ values
        row += m
    return {"out": out, "lse": lse}
