"""Refusals of the entry points for steps whose lengths live on the GPU, on the
CPU: every bad argument is turned down before a launch. The same calls run
against a build of the entry points with AddressSanitizer and UBSan."""
import ctypes
import math
import os
import subprocess
import sys

import pytest

import host_sanitizer
from paper_2607_03333_amd import spork

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, UNSUPPORTED, CAPACITY = spork.SPORK_E_INVAL, spork.SPORK_E_UNSUPPORTED, spork.SPORK_E_CAPACITY
BF16, F32 = spork.SPORK_DTYPE_BF16, spork.SPORK_DTYPE_F32
P = 1 << 20  # a pointer that nothing follows: every call here is turned down


def tables(**kw):
    f = dict(num_blocks=100, block_size=16, n_seqs=4, max_blocks=8, table=P, held=P, refcount=P, free_queue=P, queue=P)
    f.update(kw)
    return ctypes.byref(spork.spork_tables(*f.values()))


def shape(hq=32, hkv=8, d=128, bs=16, dtype=BF16, scale=0.1):
    return ctypes.byref(spork.make_shape(hq, hkv, d, bs, dtype, scale))


BAD_TABLES = [(dict(num_blocks=0), INVAL), (dict(block_size=0), INVAL), (dict(n_seqs=0), INVAL), (dict(max_blocks=-1), INVAL),
              (dict(n_seqs=1 << 16, max_blocks=1 << 15), UNSUPPORTED), (dict(block_size=1 << 20, max_blocks=1 << 11), UNSUPPORTED)]
BAD_MEMORY = [({k: None}, INVAL) for k in ("table", "held", "refcount", "free_queue", "queue")]


def step(t=None, size=1 << 20, **kw):
    f = dict(lens=P, n_new=P, parents=None, max_tokens=9, slots=P, positions=None, row_off=P, kv_len=P, copies=P, n_copies=P,
             status=P, workspace=P)
    f.update(kw)
    return spork.lib().spork_tables_step(t or tables(), *f.values(), size, None)


@pytest.mark.parametrize("fields,code", BAD_TABLES + BAD_MEMORY)
def test_tables_of_bad_sizes_and_memory(fields, code):
    lib, b = spork.lib(), ctypes.c_size_t(77)
    assert step(tables(**fields)) == code
    assert lib.spork_tables_init(tables(**fields), None, None) == code
    if (fields, code) in BAD_TABLES:
        assert lib.spork_tables_workspace_bytes(tables(**fields), ctypes.byref(b)) == code and b.value == 77
        assert lib.spork_tables_workspace_clear(tables(**fields), P, 1 << 20, None) == code
    assert spork.lib().spork_last_error()


def test_tables_arguments():
    lib, b = spork.lib(), ctypes.c_size_t()
    for name in ("lens", "n_new", "slots", "row_off", "kv_len", "copies", "n_copies", "status", "workspace"):
        assert step(**{name: None}) == INVAL, name
    assert step(max_tokens=-1) == INVAL and step(workspace=P + 16) == INVAL
    assert lib.spork_tables_workspace_bytes(tables(), ctypes.byref(b)) == 0
    assert step(size=b.value - 1) == CAPACITY
    assert lib.spork_tables_workspace_clear(tables(), P, b.value - 1, None) == CAPACITY
    assert lib.spork_tables_workspace_clear(tables(), None, b.value, None) == INVAL
    for f in (lib.spork_tables_init, lib.spork_tables_workspace_clear):
        assert (f(None, None, None) if f is lib.spork_tables_init else f(None, P, 1 << 20, None)) == INVAL
    assert lib.spork_tables_workspace_bytes(None, ctypes.byref(b)) == INVAL
    assert lib.spork_tables_workspace_bytes(tables(), None) == INVAL
    assert lib.spork_tables_step(None, *[P] * 3, 9, *[P] * 8, 1 << 20, None) == INVAL


def test_steps_larger_than_a_launch():
    """Threads of a launch are counted in 32 bits: refused before anything is launched."""
    many = dict(n_seqs=1 << 24, max_blocks=1)
    assert step(tables(**many), size=1 << 40) == UNSUPPORTED
    assert step(tables(n_seqs=(1 << 24) - 2, max_blocks=1), max_tokens=300, size=1 << 40) == UNSUPPORTED
    assert step(tables(n_seqs=1 << 30, max_blocks=1), size=1 << 40) == UNSUPPORTED  # takes of two blocks a row: 2^31
    call = spork.lib().spork_kv_copy_batch
    assert call(shape(hq=8, hkv=8), P, P, 10, P, P, 1 << 21, None) == UNSUPPORTED


def test_copy_batch_arguments():
    call = spork.lib().spork_kv_copy_batch
    assert call(shape(), P, P, 10, P, P, 0, None) == 0  # nothing to copy
    for i in (1, 2, 4, 5):
        args = [shape(), P, P, 10, P, P, 3, None]
        args[i] = None
        assert call(*args) == INVAL, i
    assert call(None, P, P, 10, P, P, 3, None) == INVAL
    assert call(shape(), P, P, 0, P, P, 3, None) == INVAL and call(shape(), P, P, 10, P, P, -1, None) == INVAL
    assert call(shape(), P + 8, P, 10, P, P, 3, None) == INVAL and call(shape(), P, P + 4, 10, P, P, 3, None) == INVAL
    assert call(shape(d=12), P, P, 10, P, P, 3, None) == UNSUPPORTED
    assert call(shape(hq=2, hkv=2, d=6, dtype=F32), P, P, 10, P, P, 3, None) == UNSUPPORTED
    assert call(shape(), P, P, 10, P, P, 1 << 29, None) == UNSUPPORTED
    assert call(shape(d=1 << 20, bs=1 << 11), P, P, 10, P, P, 3, None) == UNSUPPORTED
    assert call(shape(dtype=7), P, P, 10, P, P, 3, None) == UNSUPPORTED
    assert call(shape(hq=3, hkv=2), P, P, 10, P, P, 3, None) == INVAL


def chunk(sh=None, size=1 << 30, **kw):
    f = dict(q=P, q_stride=32 * 128, k=P, v=P, num_blocks=9, table=P, max_blocks=5, row_off=P, kv_len=P, n_seqs=3, n_rows=7,
             out=P, lse=None, workspace=P)
    f.update(kw)
    return spork.lib().spork_chunk_attn(sh or shape(), *f.values(), size, None)


@pytest.mark.parametrize("bad,code", [
    (dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(bs=8), UNSUPPORTED), (dict(bs=64), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(hq=257, hkv=1), UNSUPPORTED), (dict(hq=30), INVAL), (dict(hkv=0), INVAL),
    (dict(scale=math.inf), INVAL), (dict(scale=math.nan), INVAL)])
def test_chunk_shapes(bad, code):
    b = ctypes.c_size_t(77)
    assert chunk(shape(**bad)) == code
    assert spork.lib().spork_chunk_workspace_bytes(shape(**bad), 1, 1, ctypes.byref(b)) == code and b.value == 77


def test_chunk_arguments():
    lib, b = spork.lib(), ctypes.c_size_t()
    for name in ("q", "k", "v", "table", "row_off", "kv_len", "out", "workspace"):
        assert chunk(**{name: None}) == INVAL, name
    for name in ("q", "k", "v", "out"):
        assert chunk(**{name: P + 8}) == INVAL, name
    assert chunk(workspace=P + 128) == INVAL
    for bad in (dict(n_seqs=-1), dict(n_rows=-1), dict(num_blocks=0), dict(max_blocks=0), dict(q_stride=32 * 128 - 8),
                dict(q_stride=-32 * 128), dict(q_stride=32 * 128 + 4), dict(q_stride=1 << 61)):
        assert chunk(**bad) == INVAL, bad
    assert chunk(shape(dtype=F32), q_stride=32 * 128 + 2) == INVAL
    assert chunk(max_blocks=1 << 27) == UNSUPPORTED
    assert chunk(shape(scale=3e38)) == INVAL
    assert chunk(n_seqs=0) == 0 and chunk(n_rows=0, q=None, out=None, workspace=None, size=0) == 0  # nothing to do
    assert lib.spork_chunk_workspace_bytes(shape(), 3, 7, ctypes.byref(b)) == 0
    assert chunk(size=b.value - 1) == CAPACITY
    for bad in ((None, 1, 1, ctypes.byref(b)), (shape(), 1, 1, None), (shape(), -1, 1, ctypes.byref(b)), (shape(), 1, -1, ctypes.byref(b))):
        assert lib.spork_chunk_workspace_bytes(*bad) == INVAL
    assert lib.spork_chunk_workspace_bytes(shape(), 0, 9, ctypes.byref(b)) == 0 and b.value == 0


def test_binding_checks_what_it_hands_over():
    torch = pytest.importorskip("torch")
    i32 = lambda *m: torch.zeros(m, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        spork.make_tables(16, i32(2, 4), i32(3), i32(9), i32(9), i32(2))
    with pytest.raises(ValueError):
        spork.make_tables(16, i32(2, 4), i32(2).long(), i32(9), i32(9), i32(2))
    t = spork.make_tables(16, i32(2, 4), i32(2), i32(9), i32(9), i32(2))
    good = [i32(2), i32(2), None, torch.zeros(5, dtype=torch.int64), i32(5), i32(3), i32(2), i32(2, 3), i32(1), i32(1),
            torch.zeros(1 << 12, dtype=torch.uint8)]
    for i, wrong in ((0, i32(3)), (2, i32(1)), (3, i32(5)), (4, i32(4)), (5, i32(2)), (7, i32(2)), (8, i32(2)), (9, i32(0))):
        args = list(good)
        args[i] = wrong
        with pytest.raises(ValueError) as e:
            spork.spork_tables_step(t, *args, stream=0)
        assert "GPU" not in str(e.value)
    with pytest.raises(ValueError, match="GPU"):  # host tensors
        spork.spork_tables_step(t, *good, stream=0)
    with pytest.raises(ValueError, match="GPU"):
        spork.spork_tables_init(t, stream=0)
    with pytest.raises(ValueError, match="GPU"):
        spork.spork_tables_workspace_clear(t, torch.zeros(1 << 12, dtype=torch.uint8), stream=0)
    sh = spork.make_shape(4, 2, 64, 16, F32, 0.1)
    q, k, v = torch.zeros(3, 4, 64), torch.zeros(5, 2, 16, 64), torch.zeros(5, 2, 64, 16)
    good = [q, k, v, i32(2, 4), i32(3), i32(2), torch.zeros(3, 4, 64), torch.zeros(3, 4), torch.zeros(64)]
    for i, wrong in ((0, q[:, :3]), (0, q.half()), (0, torch.zeros(3, 4, 128)[..., ::2]), (1, v), (2, k), (2, v[:4]), (4, i32(2)),
                     (5, i32(3)), (5, i32(2).float()), (6, q[:2]), (7, torch.zeros(3, 3)), (7, torch.zeros(3, 4).half()),
                     (3, i32(4, 2).t())):
        args = list(good)
        args[i] = wrong
        with pytest.raises(ValueError) as e:
            spork.spork_chunk_attn(sh, *args, stream=0)
        assert "GPU" not in str(e.value)
    with pytest.raises(ValueError, match="GPU"):
        spork.spork_chunk_attn(sh, *good, stream=0)
    with pytest.raises(ValueError, match="GPU"):
        spork.spork_kv_copy_batch(sh, k, v, 5, i32(2, 3), i32(1), stream=0)


def test_entry_points_are_clean_under_asan_and_ubsan():
    if os.environ.get("SPORK_HOST_SANITIZER_LIB"):
        pytest.skip("runs inside the sanitizer build already")
    csrc = host_sanitizer.CSRC
    out = os.path.join(ROOT, "_build", "libspork_paged_asan.so")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
           f"-I{os.path.join(host_sanitizer.ROCM, 'include')}", f"-I{os.path.join(ROOT, 'include')}", f"-I{csrc}",
           *host_sanitizer.SOURCES, os.path.join(csrc, "paged.cpp"), os.path.join(ROOT, "tests", "paged_stubs.cpp"),
           "-o", out, f"-L{os.path.join(host_sanitizer.ROCM, 'lib')}", "-lamdhip64",
           f"-Wl,-rpath,{os.path.join(host_sanitizer.ROCM, 'lib')}"]
    os.makedirs(os.path.dirname(out), exist_ok=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    env = dict(os.environ)
    env.update(LD_PRELOAD=host_sanitizer.runtime_preload(), SPORK_HOST_SANITIZER_LIB=out,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-p", "no:cacheprovider"], cwd=ROOT,
                       env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert "AddressSanitizer" not in r.stdout and "runtime error" not in r.stdout, r.stdout[-3000:]
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:]
