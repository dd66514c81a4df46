"""Refusals of the entry points between a projection's rows and the cache, and the
frequencies of rotary positions, on the CPU: every bad argument is turned down
before a launch. The same calls run against a build of the entry points with
AddressSanitizer and UBSan."""
import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest

import host_sanitizer
from paper_2607_03333_amd import spork

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, UNSUPPORTED, CAPACITY = spork.SPORK_E_INVAL, spork.SPORK_E_UNSUPPORTED, spork.SPORK_E_CAPACITY
BF16, F32 = spork.SPORK_DTYPE_BF16, spork.SPORK_DTYPE_F32
P = 1 << 20  # a pointer that nothing follows: every call here is turned down


def at(i):
    """Pointers 64 MiB apart, so that the rows behind them are apart."""
    return (i + 1) << 26


def shape(hq=32, hkv=8, d=128, bs=16, dtype=BF16, scale=0.1):
    return ctypes.byref(spork.make_shape(hq, hkv, d, bs, dtype, scale))


def rope(rotary=128, layout=0, magnitude=1.0, freq=P):
    return ctypes.byref(spork.spork_rope(rotary, layout, magnitude, freq))


def norm(q=P, k=P, eps=1e-6):
    return ctypes.byref(spork.spork_qk_norm(q, k, eps))


def kvq(**kw):
    f = dict(num_blocks=100, k_codes=at(10), v_codes=at(11), k_scale=at(12), v_scale=at(13))
    f.update(kw)
    return ctypes.byref(spork.spork_kvq(*f.values()))


def turn(sh=None, **kw):
    f = dict(rope=rope(), norm=norm(), positions=P, n_rows=7, q=at(0), q_stride=32 * 128, k=at(1), k_stride=8 * 128, q_out=at(2),
             q_out_stride=32 * 128, k_out=at(3), k_out_stride=8 * 128)
    f.update(kw)
    return spork.lib().spork_qk_rope(sh or shape(), *f.values(), None)


def write(sh=None, **kw):
    f = dict(cache=kvq(), rope=rope(), norm=norm(), slots=P, positions=P, n_rows=7, q=at(0), q_stride=32 * 128, k=at(1),
             k_stride=8 * 128, v=at(2), v_stride=8 * 128, q_out=at(3), q_out_stride=32 * 128, bad=None)
    f.update(kw)
    return spork.lib().spork_kvq_write(sh or shape(), *f.values(), None)


def attn(sh=None, size=1 << 30, **kw):
    f = dict(q=P, q_stride=32 * 128, cache=kvq(), table=P, max_blocks=5, row_off=P, kv_len=P, n_seqs=3, n_rows=7, out=P, lse=None,
             workspace=P)
    f.update(kw)
    return spork.lib().spork_kvq_attn(sh or shape(), *f.values(), size, None)


def copy(sh=None, cache=None, copies=P, n_copies=P, most=3):
    return spork.lib().spork_kvq_copy_batch(sh or shape(), cache or kvq(), copies, n_copies, most, None)


BAD_SHAPES = [(dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(hq=30), INVAL),
              (dict(hkv=0), INVAL), (dict(scale=math.inf), INVAL), (dict(hq=1 << 25, hkv=1), UNSUPPORTED)]
BAD_BLOCKS = [(dict(bs=8), UNSUPPORTED), (dict(bs=64), UNSUPPORTED), (dict(bs=0), INVAL)]


@pytest.mark.parametrize("bad,code", BAD_SHAPES + BAD_BLOCKS)
def test_shapes(bad, code):
    assert write(shape(**bad)) == code and attn(shape(**bad)) == code and copy(shape(**bad)) == code
    if (bad, code) in BAD_SHAPES:
        assert turn(shape(**bad)) == code
    assert spork.lib().spork_last_error()


@pytest.mark.parametrize("call", (turn, write))
def test_rotations_and_norms(call):
    for bad, code in [(dict(rotary=0), UNSUPPORTED), (dict(rotary=8), UNSUPPORTED), (dict(rotary=24), UNSUPPORTED),
                      (dict(rotary=144), UNSUPPORTED), (dict(rotary=-16), UNSUPPORTED), (dict(layout=2), INVAL),
                      (dict(layout=-1), INVAL), (dict(magnitude=math.nan), INVAL), (dict(magnitude=-math.inf), INVAL),
                      (dict(freq=None), INVAL), (dict(freq=P + 8), INVAL)]:
        assert call(rope=rope(**bad)) == code, bad
    assert call(shape(d=64, hq=64, hkv=16), rope=rope(128)) == UNSUPPORTED
    for bad in (dict(q=None), dict(k=None), dict(q=P + 2), dict(k=P + 8), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf)):
        assert call(norm=norm(**bad)) == INVAL, bad
    assert call(positions=None) == INVAL
    assert call(n_rows=-1) == INVAL
    assert call(n_rows=0, q=None, k=None) == 0  # nothing to do
    assert call(None) is not None and spork.lib().spork_qk_rope(None, *[None] * 3, 1, *[None, 0] * 4, None) == INVAL


def test_rows_of_a_rotation():
    assert turn(rope=None, norm=None) == INVAL and turn(q=None, q_out=None, k=None, k_out=None) == INVAL
    for name in ("q", "k", "q_out", "k_out"):
        for bad in ({name: None}, {name: at(20) + 8}, {name + "_stride": 8 * 128 - 8}, {name + "_stride": -4096},
                    {name + "_stride": 32 * 128 + 4}, {name + "_stride": 1 << 61}):
            assert turn(**bad) == INVAL, bad
    assert turn(shape(dtype=F32), q_stride=32 * 128 + 2) == INVAL
    assert turn(n_rows=1 << 25, q_out=1 << 50, k=None, k_out=None) == UNSUPPORTED


def test_outputs_apart_from_inputs():
    """Rows of bf16, 32 query and 8 KV heads of 128, of strides of their own or inside rows of `wide`: whatever meets what is
    read or the other output is refused, but for an output in its input's place."""
    q, k, wide = 4096, 1024, 6 * 1024
    overlaps = [dict(q_out=at(0) + 256), dict(q_out=at(0) + 2 * q), dict(q_out=at(4)), dict(k_out=at(0)), dict(k_out=at(6)),
                dict(q_out=at(0), q_out_stride=q + 8), dict(k_out=at(4), k_out_stride=2 * k),
                dict(q_stride=wide, q_out=at(0) + 2 * 2048, q_out_stride=wide),
                dict(q_stride=wide, k=at(0) + 2 * q, k_stride=wide, q_out=at(0), q_out_stride=wide, k_out=at(0) + 2 * (q - 8), k_out_stride=wide),
                dict(q_out_stride=wide, k_out=at(6) + 2 * (wide - 512), k_out_stride=wide),
                dict(q_stride=wide, k=at(0) + 2 * q, k_stride=wide, q_out=at(0) + 2 * (q + k), q_out_stride=q + 8)]
    for bad in overlaps:
        f = dict(q=at(0), q_stride=q, k=at(4), k_stride=k, q_out=at(6), q_out_stride=q, k_out=at(9), k_out_stride=k, n_rows=6000)
        assert turn(**{**f, **bad}) == INVAL and b"overlap" in spork.lib().spork_last_error(), bad


def test_rows_of_a_write():
    assert write(rope=None, norm=None) == INVAL  # queries that nothing happens to
    for name in ("q", "k", "v", "q_out"):
        for bad in ({name: None}, {name: at(20) + 8}, {name + "_stride": 8 * 128 - 8}, {name + "_stride": -4096},
                    {name + "_stride": 32 * 128 + 4}, {name + "_stride": 1 << 61}):
            assert write(**bad) == INVAL, bad
    assert write(slots=None) == INVAL
    for bad in (dict(num_blocks=0), dict(k_codes=None), dict(v_codes=None), dict(k_scale=None), dict(v_scale=None),
                dict(k_codes=P + 8), dict(v_codes=P + 4)):
        assert write(cache=kvq(**bad)) == INVAL and attn(cache=kvq(**bad)) == INVAL and copy(cache=kvq(**bad)) == INVAL, bad
    assert write(cache=None) == INVAL and attn(cache=None) == INVAL
    assert spork.lib().spork_kvq_copy_batch(shape(), None, P, P, 3, None) == INVAL
    for bad in (dict(q_out=at(0) + 256), dict(q_out=at(1)), dict(q_out=at(2) + 512), dict(q_out=at(0), q_out_stride=8192)):
        assert write(**bad) == INVAL and b"overlap" in spork.lib().spork_last_error(), bad
    assert write(n_rows=1 << 20, q=None, q_out=None, norm=None) == UNSUPPORTED
    for heads in (dict(hq=1, hkv=1, d=64), dict(hq=1 << 15, hkv=1 << 15, d=64, bs=32)):  # the fewest and the most KV heads
        wide, most = heads["hq"] * 64, (1 << 25) // (heads["hq"] + heads["hkv"])
        f = dict(rope=None, norm=None, q=None, q_out=None, q_stride=0, q_out_stride=0, k_stride=wide, v=1 << 50, v_stride=wide)
        assert write(shape(**heads), n_rows=most, **f) == UNSUPPORTED and b"2^25" in spork.lib().spork_last_error()


def test_blocks_of_many_heads():
    """A block's codes of all heads are placed by 31 bits."""
    for d, bs, hkv in ((64, 16, 1 << 21), (128, 32, 1 << 19)):
        for call in (write, attn, copy):
            assert call(shape(hq=hkv, hkv=hkv, d=d, bs=bs)) == UNSUPPORTED, (call, d)
            assert b"2^31" in spork.lib().spork_last_error()


def test_copies():
    assert copy(most=0, copies=None, n_copies=None) == 0  # nothing to copy
    assert copy(copies=None) == INVAL and copy(n_copies=None) == INVAL and copy(most=-1) == INVAL
    assert copy(most=1 << 21) == UNSUPPORTED and copy(shape(hq=1 << 12, hkv=1 << 12, d=64), most=1 << 12) == UNSUPPORTED


def test_attention_arguments():
    b = ctypes.c_size_t()
    for name in ("q", "table", "row_off", "kv_len", "out", "workspace"):
        assert attn(**{name: None}) == INVAL, name
    assert attn(q=P + 8) == INVAL and attn(out=P + 8) == INVAL and attn(workspace=P + 128) == INVAL
    for bad in (dict(n_seqs=-1), dict(n_rows=-1), dict(max_blocks=0), dict(q_stride=32 * 128 - 8), dict(q_stride=-32 * 128),
                dict(q_stride=32 * 128 + 4), dict(q_stride=1 << 61)):
        assert attn(**bad) == INVAL, bad
    assert attn(max_blocks=1 << 27) == UNSUPPORTED and attn(shape(bs=32), max_blocks=((1 << 31) - 4096) // 32) == UNSUPPORTED
    assert attn(shape(hq=257, hkv=1)) == UNSUPPORTED and attn(shape(scale=3e38)) == INVAL
    assert attn(n_seqs=0) == 0 and attn(n_rows=0, q=None, out=None, workspace=None, size=0) == 0  # nothing to do
    if not os.environ.get("SPORK_HOST_SANITIZER_LIB"):
        assert spork.lib().spork_chunk_workspace_bytes(shape(), 3, 7, ctypes.byref(b)) == 0
        assert attn(size=b.value - 1) == CAPACITY
    assert attn(size=1000) == CAPACITY
    row = 32 * 128 * 2
    for bad in (dict(out=at(0)), dict(out=at(0) + 6 * row), dict(out=at(0) - 6 * row), dict(q_stride=48 * 128, out=at(0) + 32 * 128 * 2)):
        assert attn(**{**dict(q=at(0)), **bad}) == INVAL and b"overlap" in spork.lib().spork_last_error(), bad


def test_plain_frequencies():
    for rotary, base in ((2, 10.0), (16, 10000.0), (64, 5e5), (128, 1e6)):
        freq, magnitude = spork.spork_rope_frequencies(rotary, base)
        assert magnitude == 1.0 and len(freq) == rotary // 2
        np.testing.assert_allclose(freq, base ** (-2.0 * np.arange(rotary // 2) / rotary), rtol=1e-14)


def _scaling(kind, trained=0, factor=4.0, fast=0.0, slow=0.0):
    return spork.spork_rope_scaling(kind, trained, factor, fast, slow)


def test_scaled_frequencies():
    """Each scaling by what it is for: which pairs keep their frequency, which are stretched, and what lies between."""
    rotary, base, trained = 128, 1e6, 32768
    plain, _ = spork.spork_rope_frequencies(rotary, base)
    turns = trained * plain / (2 * math.pi)
    got, m = spork.spork_rope_frequencies(rotary, base, _scaling(spork.SPORK_ROPE_SCALE_LINEAR, factor=8.0))
    np.testing.assert_allclose(got, plain / 8, rtol=1e-15)
    assert m == 1.0
    got, m = spork.spork_rope_frequencies(rotary, base, _scaling(spork.SPORK_ROPE_SCALE_BASE, factor=8.0))
    assert m == 1.0 and got[0] == 1.0  # the fastest pair as it was, the slowest stretched by the whole factor
    np.testing.assert_allclose(got[-1], plain[-1] / 8, rtol=1e-12)
    got, m = spork.spork_rope_frequencies(rotary, base, _scaling(spork.SPORK_ROPE_SCALE_BANDS, trained, 8.0, 4.0, 1.0))
    assert m == 1.0
    np.testing.assert_allclose(got[turns >= 4], plain[turns >= 4], rtol=1e-15)
    np.testing.assert_allclose(got[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    keep = (turns[between] - 1) / 3
    np.testing.assert_allclose(got[between], plain[between] * (keep + (1 - keep) / 8), rtol=1e-13)
    got, m = spork.spork_rope_frequencies(rotary, base, _scaling(spork.SPORK_ROPE_SCALE_PARTS, trained, 4.0, 32.0, 1.0))
    assert m == 0.1 * math.log(4.0) + 1
    index = lambda t: math.log(trained / (t * 2 * math.pi)) / math.log(base) * rotary / 2  # noqa: E731 the pair that makes t turns
    low, high = math.floor(index(32)), math.ceil(index(1))
    np.testing.assert_allclose(got[:low + 1], plain[:low + 1], rtol=1e-15)
    np.testing.assert_allclose(got[high:], plain[high:] / 4, rtol=1e-15)
    i = np.arange(low, high + 1)
    np.testing.assert_allclose(got[i], plain[i] * (1 - (i - low) / (high - low) * 0.75), rtol=1e-13)
    # nothing is stretched, nothing is left: both ends of the pairs
    got, m = spork.spork_rope_frequencies(16, 10.0, _scaling(spork.SPORK_ROPE_SCALE_PARTS, 1 << 30, 1.0, 32.0, 1.0))
    np.testing.assert_allclose(got, spork.spork_rope_frequencies(16, 10.0)[0], rtol=1e-15)
    assert m == 1.0
    got, _ = spork.spork_rope_frequencies(16, 10.0, _scaling(spork.SPORK_ROPE_SCALE_PARTS, 1, 2.0, 32.0, 1.0))
    assert (got <= spork.spork_rope_frequencies(16, 10.0)[0]).all() and (got > 0).all()


def test_frequencies_are_refused():
    f, m = (ctypes.c_double * 64)(), ctypes.c_double(7)
    call = spork.lib().spork_rope_frequencies
    for bad in ((0, 1e4), (-2, 1e4), (7, 1e4), (64, 1.0), (64, -3.0), (64, math.inf), (64, math.nan)):
        assert call(*bad, None, f, ctypes.byref(m)) == INVAL, bad
    assert call(64, 1e4, None, None, ctypes.byref(m)) == INVAL and call(64, 1e4, None, f, None) == INVAL
    for s in (_scaling(0), _scaling(5), _scaling(1, factor=0.0), _scaling(1, factor=math.nan), _scaling(3, 0, 2.0, 32.0, 1.0),
              _scaling(3, 10, 2.0, 1.0, 1.0), _scaling(4, 10, 2.0, 4.0, 0.0), _scaling(4, 10, 2.0, math.inf, 1.0),
              _scaling(4, 10, 2.0, 4.0, math.nan), _scaling(3, 10, 2.0, math.nan, 1.0)):
        assert call(64, 1e4, ctypes.byref(s), f, ctypes.byref(m)) == INVAL
    assert call(2, 1e4, ctypes.byref(_scaling(spork.SPORK_ROPE_SCALE_BASE)), f, ctypes.byref(m)) == INVAL
    assert m.value == 7


def test_binding_checks_what_it_hands_over():
    torch = pytest.importorskip("torch")
    i32 = lambda *m: torch.zeros(m, dtype=torch.int32)  # noqa: E731
    sh = spork.make_shape(4, 2, 64, 16, F32, 0.1)
    for bad in (torch.zeros(32), torch.zeros(8, 4, dtype=torch.float64), torch.zeros(64, dtype=torch.float64)[::2]):
        with pytest.raises(ValueError):
            spork.make_rope(bad)
    r = spork.make_rope(torch.zeros(32, dtype=torch.float64))
    for bad in ((torch.zeros(8, 8), None), (None, torch.zeros(128)[::2])):
        with pytest.raises(ValueError):
            spork.make_qk_norm(*bad, 1e-6)
    n = spork.make_qk_norm(torch.ones(64), torch.ones(64), 1e-6)
    u8 = lambda *m: torch.zeros(m, dtype=torch.uint8)  # noqa: E731
    pools = [u8(5, 2, 16, 64), u8(5, 2, 64, 16), u8(5, 2), u8(5, 2)]
    for i, bad in ((0, u8(5, 2, 16)), (0, pools[0].float()), (1, pools[0]), (2, u8(5, 3)), (3, u8(5, 2).int()), (3, u8(2, 5).t()),
                   (0, u8(5, 2, 16, 128)[..., ::2]), (1, pools[1].view(torch.int8))):
        args = list(pools)
        args[i] = bad
        with pytest.raises(ValueError):
            spork.make_kvq(*args)
    spork.make_kvq(*(x.view(torch.float8_e4m3fn) for x in pools[:2]), *(x.view(torch.float8_e8m0fnu) for x in pools[2:]))
    c = spork.make_kvq(*pools)
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)

    def refused(call, good, wrong, *keep):
        for i, bad in wrong:
            args = list(good)
            args[i] = bad
            with pytest.raises(ValueError) as e:
                call(*keep, *args, stream=0)
            assert "GPU" not in str(e.value), (i, e.value)
        with pytest.raises(ValueError, match="GPU"):
            call(*keep, *good, stream=0)

    wide = torch.zeros(3, 4, 128)[..., ::2]
    other = spork.make_qk_norm(torch.ones(128), torch.ones(64), 1e-6)
    refused(spork.spork_qk_rope, [r, n, i32(3), q, k, q.clone(), k.clone()],
            [(2, i32(4)), (2, i32(3).float()), (3, q[:, :3]), (3, q.bfloat16()), (3, wide), (4, k[:2]), (5, k), (6, q), (6, k.half()),
             (1, other), (1, spork.make_qk_norm(torch.ones(64).half(), None, 1e-6))], sh)
    good = [c, r, n, torch.zeros(3, dtype=torch.int64), i32(3), q, k, k.clone(), q.clone(), i32(1)]
    refused(spork.spork_kvq_write, good,
            [(0, spork.make_kvq(u8(5, 2, 32, 64), u8(5, 2, 64, 32), u8(5, 2), u8(5, 2))), (2, other), (3, i32(3)), (4, i32(2)), (5, wide),
             (6, q), (7, k.double()), (8, q[:2]), (9, i32(2)), (6, torch.zeros(3, 2, 128)[..., ::2])], sh)
    refused(spork.spork_kvq_copy_batch, [c, i32(2, 3), i32(1)],
            [(0, spork.make_kvq(u8(5, 4, 16, 64), u8(5, 4, 64, 16), u8(5, 4), u8(5, 4))), (1, i32(2, 2)), (2, i32(2))], sh)
    refused(spork.spork_kvq_attn, [q, c, i32(2, 4), i32(3), i32(2), q.clone(), torch.zeros(3, 4), torch.zeros(64)],
            [(0, q[:, :3]), (0, wide), (0, q.bfloat16()), (2, i32(4, 2).t()), (3, i32(2)), (4, i32(3)), (5, q[:2].clone()),
             (5, q.half()), (6, torch.zeros(3, 3)), (6, torch.zeros(3, 4).half()),
             (1, spork.make_kvq(u8(5, 2, 16, 128), u8(5, 2, 128, 16), u8(5, 2), u8(5, 2)))], sh)


def test_entry_points_are_clean_under_asan_and_ubsan():
    if os.environ.get("SPORK_HOST_SANITIZER_LIB"):
        pytest.skip("runs inside the sanitizer build already")
    csrc = host_sanitizer.CSRC
    out = os.path.join(ROOT, "_build", "libspork_rows_asan.so")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
           f"-I{os.path.join(host_sanitizer.ROCM, 'include')}", f"-I{os.path.join(ROOT, 'include')}", f"-I{csrc}",
           *host_sanitizer.SOURCES, os.path.join(csrc, "rows.cpp"), os.path.join(ROOT, "tests", "rows_stubs.cpp"),
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
