"""Calls of the entry points for steps whose lengths live on the GPU that are
refused on the host because the kernels could not answer them: buffers that
overlap, sizes at the end of 32 bits. On the CPU; nothing is launched."""
import ctypes

import pytest

from paper_2607_03333_amd import spork

INVAL, UNSUPPORTED = spork.SPORK_E_INVAL, spork.SPORK_E_UNSUPPORTED
N, BLOCKS, MOST, TOKENS = 40, 100, 8, 64
WS = 1 << 20


def step_args(**kw):
    """A step of N rows whose buffers lie apart, 16 MiB each from the next; nothing follows the pointers."""
    names = ("table", "held", "refcount", "free_queue", "queue", "lens", "n_new", "parents", "slots", "positions", "row_off",
             "kv_len", "copies", "n_copies", "status", "workspace")
    f = {name: (i + 1) << 24 for i, name in enumerate(names)}
    f.update(kw)
    return f


def step(f):
    t = spork.spork_tables(BLOCKS, 16, N, MOST, f["table"], f["held"], f["refcount"], f["free_queue"], f["queue"])
    rc = spork.lib().spork_tables_step(ctypes.byref(t), f["lens"], f["n_new"], f["parents"], TOKENS, f["slots"], f["positions"],
                                       f["row_off"], f["kv_len"], f["copies"], f["n_copies"], f["status"], f["workspace"], WS, None)
    return rc, spork.lib().spork_last_error().decode()


INPUTS = ("lens", "n_new", "parents")
WRITTEN = {"table": 4 * N * MOST, "held": 4 * N, "refcount": 4 * BLOCKS, "free_queue": 4 * BLOCKS, "queue": 8, "slots": 8 * TOKENS,
           "positions": 4 * TOKENS, "row_off": 4 * (N + 1), "kv_len": 4 * N, "copies": 12 * N, "n_copies": 4, "status": 4}


@pytest.mark.parametrize("written", sorted(WRITTEN))
def test_what_a_step_writes_lies_apart(written):
    """The buffer itself in place of another, and its last four bytes as the first of another."""
    for other in INPUTS + tuple(w for w in WRITTEN if w != written):
        apart = step_args()
        for at in (apart[written], apart[written] + WRITTEN[written] - 4):
            rc, why = step(step_args(**{other: at}))
            assert rc == INVAL and "overlap" in why, (written, other)


def test_the_workspace_lies_apart():
    for other in INPUTS + tuple(WRITTEN):
        rc, why = step(step_args(**{other: step_args()["workspace"] + 4}))
        assert rc == INVAL and "overlap" in why, other


@pytest.mark.parametrize("block_size", (16, 32))
def test_contexts_near_the_end_of_32_bits(block_size):
    """The kernel's positions run a few stages past a context's end, in 32 bits: wider tables are refused. (Without a
    workspace, so that nothing is launched where the size is taken.)"""
    shape = ctypes.byref(spork.make_shape(8, 2, 64, block_size, spork.SPORK_DTYPE_BF16, 0.1))
    p = 1 << 20

    def call(max_blocks):
        return spork.lib().spork_chunk_attn(shape, p, 8 * 64, p, p, 9, p, max_blocks, p, p, 1, 1, p, None, None, 0, None)

    least = ((1 << 31) - 4096) // block_size
    assert [call(m) for m in (least, least + 1, (1 << 31) // block_size - 1, (1 << 31) - 1)] == [UNSUPPORTED] * 4
    assert call(least - 1) == INVAL


def test_rows_near_the_end_of_32_bits():
    """The kernels' columns run up to 1,024 entries past a row's last one, in 32 bits: wider rows are refused."""
    size = ctypes.c_size_t()

    def need(max_blocks):
        t = spork.spork_tables(9, 1, 1, max_blocks, None, None, None, None, None)
        return spork.lib().spork_tables_workspace_bytes(ctypes.byref(t), ctypes.byref(size))

    least = (1 << 31) - 4096
    assert [need(m) for m in (least, least + 1, (1 << 31) - 3)] == [UNSUPPORTED] * 3
    assert need(least - 1) == spork.SPORK_OK and size.value > 0
    f = step_args()
    t = spork.spork_tables(BLOCKS, 1, 1, least, f["table"], f["held"], f["refcount"], f["free_queue"], f["queue"])
    rc = spork.lib().spork_tables_step(ctypes.byref(t), f["lens"], f["n_new"], f["parents"], TOKENS, f["slots"], f["positions"],
                                       f["row_off"], f["kv_len"], f["copies"], f["n_copies"], f["status"], None, WS, None)
    assert rc == UNSUPPORTED
