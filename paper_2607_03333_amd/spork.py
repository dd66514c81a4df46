"""Thin ctypes binding of ``libspork.so`` (C ABI in ``include/spork.h``).

Argument marshalling only: every function has the name of the C entry point
it calls, turns torch tensors into device pointers and numpy arrays into host
pointers, and raises :class:`SporkError` on a non-zero status. Kernels run on
the given stream, or torch's current stream. Nothing here computes any part
of the method, and nothing falls back to the CPU: without the built library
every call raises.
"""

import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspork.so")
# The sanitizer test of the host code loads an AddressSanitizer/UBSan build of
# the host sources instead (its kernel launches all fail); unset otherwise.
_HOST_SANITIZER_LIB = os.environ.get("SPORK_HOST_SANITIZER_LIB")

SPORK_OK = 0
SPORK_E_INVAL = -1
SPORK_E_NOBLOCKS = -2
SPORK_E_UNSUPPORTED = -3
SPORK_E_CAPACITY = -4
SPORK_E_HIP = -5
SPORK_DTYPE_F32 = 0
SPORK_DTYPE_BF16 = 1
SPORK_ROPE_HALF = 0
SPORK_ROPE_INTERLEAVED = 1
SPORK_ROPE_SCALE_LINEAR = 1
SPORK_ROPE_SCALE_BASE = 2
SPORK_ROPE_SCALE_PARTS = 3
SPORK_ROPE_SCALE_BANDS = 4
SPORK_KERNEL_ATTN = 0
SPORK_KERNEL_MERGE = 1
SPORK_KERNEL_ARGMAX = 2
SPORK_KERNEL_ACCEPT = 3
SPORK_KERNEL_CONF_CHUNKS = 4
SPORK_KERNEL_CONF_FINAL = 5
SPORK_KERNEL_NGRAM_SCAN = 6
SPORK_KERNEL_NGRAM_DRAFTS = 7
SPORK_KERNEL_READ_CEILING = 8
SPORK_KERNEL_KINDS = 9
KERNEL_NAMES = ("attn_partial", "merge", "argmax", "accept", "conf_chunks", "conf_final", "ngram_scan",
                "ngram_drafts", "read_ceiling")

_c_i32 = ctypes.c_int32
_c_i64 = ctypes.c_int64
_p = ctypes.c_void_p
_pi32 = ctypes.POINTER(ctypes.c_int32)
_pi64 = ctypes.POINTER(ctypes.c_int64)


class SporkError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"spork status {code}: {message}")
        self.code = code


class spork_shape(ctypes.Structure):
    _fields_ = [("hq", _c_i32), ("hkv", _c_i32), ("head_dim", _c_i32),
                ("block_size", _c_i32), ("dtype", _c_i32), ("sm_scale", ctypes.c_float)]


class spork_plan_info(ctypes.Structure):
    _fields_ = [("n_threads", _c_i32), ("n_rows", _c_i32), ("n_groups", _c_i32),
                ("n_items", _c_i32), ("n_units", _c_i32), ("n_partials", _c_i32),
                ("max_row_tiles", _c_i32), ("attn_grid", _c_i32),
                ("image_bytes", ctypes.c_size_t), ("workspace_bytes", ctypes.c_size_t),
                ("shared_tokens", _c_i64), ("private_tokens", _c_i64),
                ("unique_kv_bytes", _c_i64), ("flat_kv_bytes", _c_i64), ("attn_waves", _c_i32),
                ("attn_wide", _c_i32), ("control_bytes", ctypes.c_size_t)]


class spork_tables(ctypes.Structure):
    _fields_ = [("num_blocks", _c_i32), ("block_size", _c_i32), ("n_seqs", _c_i32), ("max_blocks", _c_i32),
                ("table", _p), ("held", _p), ("refcount", _p), ("free_queue", _p), ("queue", _p)]


class spork_rope(ctypes.Structure):
    _fields_ = [("rotary_dim", _c_i32), ("layout", _c_i32), ("magnitude", ctypes.c_double), ("inv_freq", _p)]


class spork_qk_norm(ctypes.Structure):
    _fields_ = [("q_weight", _p), ("k_weight", _p), ("eps", ctypes.c_double)]


class spork_rope_scaling(ctypes.Structure):
    _fields_ = [("kind", _c_i32), ("trained_len", _c_i32), ("factor", ctypes.c_double), ("fast", ctypes.c_double),
                ("slow", ctypes.c_double)]


class spork_kvq(ctypes.Structure):
    _fields_ = [("num_blocks", _c_i32), ("k_codes", _p), ("v_codes", _p), ("k_scale", _p), ("v_scale", _p)]


_shape, _rope, _norm, _kvq = (ctypes.POINTER(x) for x in (spork_shape, spork_rope, spork_qk_norm, spork_kvq))

# name -> (restype, argtypes); every name is declared in include/spork.h
_SIGNATURES = {
    "spork_last_error": (ctypes.c_char_p, []),
    "spork_version": (ctypes.c_int, []),
    "spork_cache_create": (ctypes.c_int, [_c_i32, _c_i32, _p, ctypes.POINTER(_p)]),
    "spork_cache_destroy": (ctypes.c_int, [_p]),
    "spork_seq_new": (ctypes.c_int, [_p, _pi32]),
    "spork_seq_append": (ctypes.c_int, [_p, _c_i32, _c_i32, _p, _p, _pi32]),
    "spork_seq_append_batch": (ctypes.c_int, [_p, _p, _p, _c_i32, _p, _p, _pi32]),
    "spork_fork": (ctypes.c_int, [_p, _c_i32, _pi32]),
    "spork_seq_free": (ctypes.c_int, [_p, _c_i32]),
    "spork_seq_len": (ctypes.c_int, [_p, _c_i32, _pi32]),
    "spork_block_table": (ctypes.c_int, [_p, _c_i32, _p, _c_i32, _pi32]),
    "spork_refcount": (ctypes.c_int, [_p, _c_i32, _pi32]),
    "spork_free_blocks": (ctypes.c_int, [_p, _p, _c_i32, _pi32]),
    "spork_kv_write": (ctypes.c_int, [ctypes.POINTER(spork_shape), _p, _p, _c_i32, _p, _p, _p,
                                      _c_i32, _p, _p]),
    "spork_kv_copy": (ctypes.c_int, [ctypes.POINTER(spork_shape), _p, _p, _c_i32, _c_i32, _c_i32,
                                     _c_i32, _p]),
    "spork_plan_create": (ctypes.c_int, [_p, ctypes.POINTER(spork_shape), _p, _p, _p, _c_i32,
                                         _c_i32, ctypes.POINTER(_p)]),
    "spork_plan_destroy": (ctypes.c_int, [_p]),
    "spork_plan_get_info": (ctypes.c_int, [_p, ctypes.POINTER(spork_plan_info)]),
    "spork_plan_image": (ctypes.c_int, [_p, _p, ctypes.c_size_t]),
    "spork_plan_advance": (ctypes.c_int, [_p, _p, _p, _p]),
    "spork_workspace_clear": (ctypes.c_int, [_p, _p, ctypes.c_size_t, _p]),
    "spork_attn_decode": (ctypes.c_int, [_p, _p, _p, _p, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "spork_verify_workspace_bytes": (ctypes.c_int, [_c_i32, _c_i32, _c_i32,
                                                    ctypes.POINTER(ctypes.c_size_t)]),
    "spork_verify_accept": (ctypes.c_int, [_p, _p, _p, _p, _p, _p, _p, _p, _c_i32, _c_i32, _p,
                                           _c_i32, _c_i32, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "spork_verify_accept_noalloc": (ctypes.c_int, [_p, _p, _p, _p, _p, _p, _p, _p, _c_i32, _c_i32, _p,
                                                   _c_i32, _c_i32, _p, _p, _p, _p]),
    "spork_confidence_workspace_bytes": (ctypes.c_int, [_c_i32, _c_i32,
                                                        ctypes.POINTER(ctypes.c_size_t)]),
    "spork_probe_confidence": (ctypes.c_int, [_p, _c_i32, _c_i32, _c_i32, _p, _c_i32, ctypes.c_float,
                                              _p, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "spork_ngram_workspace_bytes": (ctypes.c_int, [_c_i32, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "spork_ngram_propose": (ctypes.c_int, [_p, _p, _c_i32, _c_i64, _c_i32, _c_i32, _c_i32, _p, _p, _p,
                                           ctypes.c_size_t, _p]),
    "spork_tables_init": (ctypes.c_int, [ctypes.POINTER(spork_tables), _p, _p]),
    "spork_tables_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(spork_tables), ctypes.POINTER(ctypes.c_size_t)]),
    "spork_tables_workspace_clear": (ctypes.c_int, [ctypes.POINTER(spork_tables), _p, ctypes.c_size_t, _p]),
    "spork_tables_step": (ctypes.c_int, [ctypes.POINTER(spork_tables), _p, _p, _p, _c_i32, _p, _p, _p, _p, _p, _p,
                                         _p, _p, ctypes.c_size_t, _p]),
    "spork_kv_copy_batch": (ctypes.c_int, [ctypes.POINTER(spork_shape), _p, _p, _c_i32, _p, _p, _c_i32, _p]),
    "spork_chunk_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(spork_shape), _c_i32, _c_i32,
                                                   ctypes.POINTER(ctypes.c_size_t)]),
    "spork_chunk_attn": (ctypes.c_int, [ctypes.POINTER(spork_shape), _p, _c_i64, _p, _p, _c_i32, _p, _c_i32, _p, _p,
                                        _c_i32, _c_i32, _p, _p, _p, ctypes.c_size_t, _p]),
    "spork_rope_frequencies": (ctypes.c_int, [_c_i32, ctypes.c_double, ctypes.POINTER(spork_rope_scaling), _p,
                                              ctypes.POINTER(ctypes.c_double)]),
    "spork_qk_rope": (ctypes.c_int, [_shape, _rope, _norm, _p, _c_i32, _p, _c_i64, _p, _c_i64, _p, _c_i64, _p, _c_i64,
                                     _p]),
    "spork_kvq_write": (ctypes.c_int, [_shape, _kvq, _rope, _norm, _p, _p, _c_i32, _p, _c_i64, _p, _c_i64, _p, _c_i64, _p,
                                       _c_i64, _p, _p]),
    "spork_kvq_copy_batch": (ctypes.c_int, [_shape, _kvq, _p, _p, _c_i32, _p]),
    "spork_kvq_attn": (ctypes.c_int, [_shape, _p, _c_i64, _kvq, _p, _c_i32, _p, _p, _c_i32, _c_i32, _p, _p, _p,
                                      ctypes.c_size_t, _p]),
    "spork_read_ceiling": (ctypes.c_int, [_p, _c_i64, _c_i32, _c_i32, _p, _p]),
    "spork_timing_enable": (ctypes.c_int, [_c_i32]),
    "spork_timing_read": (ctypes.c_int, [_p, _p]),
}

_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        path = _HOST_SANITIZER_LIB or LIB_PATH
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with "
                               "`python -m paper_2607_03333_amd.build` (there is no fallback)")
        handle = ctypes.CDLL(path)
        for name, (res, args) in _SIGNATURES.items():
            # the sanitizer build holds only the host sources that it was given
            if _HOST_SANITIZER_LIB and not hasattr(handle, name):
                continue
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(rc):
    if rc != SPORK_OK:
        raise SporkError(rc, lib().spork_last_error().decode())


def _ptr(x):
    """Device pointer of a torch tensor, host pointer of a numpy array, or NULL."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("numpy arguments must be C-contiguous")
        return x.ctypes.data
    if not x.is_contiguous():
        raise ValueError("tensor arguments must be contiguous")
    return x.data_ptr()


_raw_stream = _raw_stream_at = None


def _stream(stream):
    global _raw_stream, _raw_stream_at
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()  # (initialises the GPU, or says why it can't)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # without a Stream object: 0.5 us against 2.9
        _raw_stream = (lambda: raw(torch.cuda.current_device())) if raw else lambda: torch.cuda.current_stream().cuda_stream
        _raw_stream_at = raw
    return _raw_stream()


def _stream_at(stream, here):
    """_stream where the current device is known."""
    return _raw_stream_at(here) if stream is None and _raw_stream_at is not None else _stream(stream)


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def make_shape(hq, hkv, head_dim, block_size, dtype, sm_scale):
    return spork_shape(hq, hkv, head_dim, block_size, dtype, sm_scale)


# ---- block manager ------------------------------------------------------------
def spork_version():
    return lib().spork_version()


def spork_cache_create(num_blocks, block_size, free_order=None):
    out = _p()
    order = None if free_order is None else _i32(free_order)
    _check(lib().spork_cache_create(num_blocks, block_size, _ptr(order), ctypes.byref(out)))
    return out


def spork_cache_destroy(cache):
    _check(lib().spork_cache_destroy(cache))


def spork_seq_new(cache):
    s = _c_i32()
    _check(lib().spork_seq_new(cache, ctypes.byref(s)))
    return s.value


def spork_seq_append(cache, seq, n_tokens):
    """Returns (slots int64 array, list of (src, dst, n_valid) copies)."""
    slots = np.zeros(max(n_tokens, 1), dtype=np.int64)
    cow = np.zeros(3, dtype=np.int32)
    n_cow = _c_i32()
    _check(lib().spork_seq_append(cache, seq, n_tokens, _ptr(slots), _ptr(cow), ctypes.byref(n_cow)))
    return slots[:n_tokens], ([tuple(int(x) for x in cow)] if n_cow.value else [])


def spork_seq_append_batch(cache, seqs, n_tokens):
    """Returns (slots int64 array in batch order, list of (src, dst, n_valid) copies)."""
    seqs, n_tokens = _i32(seqs), _i32(n_tokens)
    slots = np.zeros(max(int(np.maximum(n_tokens, 0).sum()), 1), dtype=np.int64)
    cow = np.zeros(max(3 * len(seqs), 3), dtype=np.int32)
    n_cow = _c_i32()
    _check(lib().spork_seq_append_batch(cache, _ptr(seqs), _ptr(n_tokens), len(seqs), _ptr(slots), _ptr(cow),
                                        ctypes.byref(n_cow)))
    return slots[:int(np.maximum(n_tokens, 0).sum())], [tuple(int(x) for x in cow[3 * i:3 * i + 3])
                                                        for i in range(n_cow.value)]


def spork_fork(cache, parent_seq):
    c = _c_i32()
    _check(lib().spork_fork(cache, parent_seq, ctypes.byref(c)))
    return c.value


def spork_seq_free(cache, seq):
    _check(lib().spork_seq_free(cache, seq))


def spork_seq_len(cache, seq):
    n = _c_i32()
    _check(lib().spork_seq_len(cache, seq, ctypes.byref(n)))
    return n.value


def spork_block_table(cache, seq):
    n = _c_i32()
    rc = lib().spork_block_table(cache, seq, None, 0, ctypes.byref(n))
    if rc not in (SPORK_OK, SPORK_E_CAPACITY):
        _check(rc)
    out = np.zeros(max(n.value, 1), dtype=np.int32)
    _check(lib().spork_block_table(cache, seq, _ptr(out), n.value, ctypes.byref(n)))
    return out[: n.value]


def spork_refcount(cache, block):
    r = _c_i32()
    _check(lib().spork_refcount(cache, block, ctypes.byref(r)))
    return r.value


def spork_free_blocks(cache):
    n = _c_i32()
    rc = lib().spork_free_blocks(cache, None, 0, ctypes.byref(n))
    if rc not in (SPORK_OK, SPORK_E_CAPACITY):
        _check(rc)
    out = np.zeros(max(n.value, 1), dtype=np.int32)
    _check(lib().spork_free_blocks(cache, _ptr(out), n.value, ctypes.byref(n)))
    return out[: n.value]


# ---- KV writes --------------------------------------------------------------
def spork_kv_write(shape, k_cache, v_cache, num_blocks, slots, k_new, v_new, bad_slots=None,
                   stream=None):
    _check(lib().spork_kv_write(ctypes.byref(shape), _ptr(k_cache), _ptr(v_cache), num_blocks,
                                _ptr(slots), _ptr(k_new), _ptr(v_new), int(slots.numel()),
                                _ptr(bad_slots), _stream(stream)))


def spork_kv_copy(shape, k_cache, v_cache, num_blocks, src_block, dst_block, n_valid, stream=None):
    _check(lib().spork_kv_copy(ctypes.byref(shape), _ptr(k_cache), _ptr(v_cache), num_blocks,
                               src_block, dst_block, n_valid, _stream(stream)))


# ---- plan -------------------------------------------------------------------
def spork_plan_create(cache, shape, seqs, n_rows, groups, n_cu=0):
    seqs, n_rows, groups = _i32(seqs), _i32(n_rows), _i32(groups)
    if not (len(seqs) == len(n_rows) == len(groups)):
        raise ValueError("seqs, n_rows and groups must have one entry per thread")
    out = _p()
    _check(lib().spork_plan_create(cache, ctypes.byref(shape), _ptr(seqs), _ptr(n_rows), _ptr(groups),
                                   len(seqs), n_cu, ctypes.byref(out)))
    return out


def spork_plan_destroy(plan):
    _check(lib().spork_plan_destroy(plan))


def spork_plan_get_info(plan):
    info = spork_plan_info()
    _check(lib().spork_plan_get_info(plan, ctypes.byref(info)))
    return {name: getattr(info, name) for name, _ in spork_plan_info._fields_}


def spork_plan_advance(plan, cache, dev_image, stream=None):
    _check(lib().spork_plan_advance(plan, cache, _ptr(dev_image), _stream(stream)))


def spork_plan_image(plan):
    n = spork_plan_get_info(plan)["image_bytes"]
    img = np.zeros(max(n, 1), dtype=np.uint8)
    _check(lib().spork_plan_image(plan, _ptr(img), img.nbytes))
    return img[:n]


# ---- hot path ---------------------------------------------------------------
def spork_workspace_clear(plan, workspace, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().spork_workspace_clear(plan, _ptr(workspace), ws_bytes, _stream(stream)))


def spork_attn_decode(plan, dev_image, q, k_cache, v_cache, out, lse, workspace, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().spork_attn_decode(plan, _ptr(dev_image), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                   _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream(stream)))


def spork_verify_workspace_bytes(n_verify, k_drafts, vocab):
    b = ctypes.c_size_t()
    _check(lib().spork_verify_workspace_bytes(n_verify, k_drafts, vocab, ctypes.byref(b)))
    return b.value


def spork_verify_accept(plan, dev_image, q, k_cache, v_cache, out, lse, logits, logits_dtype, vocab,
                        drafts, n_verify, k_drafts, accept_len, next_token, argmax_out, workspace,
                        stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().spork_verify_accept(plan, _ptr(dev_image), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                     _ptr(out), _ptr(lse), _ptr(logits), logits_dtype, vocab,
                                     _ptr(drafts), n_verify, k_drafts, _ptr(accept_len),
                                     _ptr(next_token), _ptr(argmax_out), _ptr(workspace), ws_bytes,
                                     _stream(stream)))


def spork_verify_accept_noalloc(plan, dev_image, q, k_cache, v_cache, out, lse, logits, logits_dtype, vocab,
                                drafts, n_verify, k_drafts, accept_len, next_token, argmax_out, stream=None):
    _check(lib().spork_verify_accept_noalloc(plan, _ptr(dev_image), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                             _ptr(out), _ptr(lse), _ptr(logits), logits_dtype, vocab,
                                             _ptr(drafts), n_verify, k_drafts, _ptr(accept_len),
                                             _ptr(next_token), _ptr(argmax_out), _stream(stream)))


def spork_confidence_workspace_bytes(n_rows, vocab):
    b = ctypes.c_size_t()
    _check(lib().spork_confidence_workspace_bytes(n_rows, vocab, ctypes.byref(b)))
    return b.value


def spork_probe_confidence(logits, logits_dtype, vocab, n_rows, span_off, n_probes, theta,
                           argmax_out, logprob_out, confidence_out, commit_out, workspace, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().spork_probe_confidence(_ptr(logits), logits_dtype, vocab, n_rows, _ptr(span_off),
                                        n_probes, float(theta), _ptr(argmax_out), _ptr(logprob_out),
                                        _ptr(confidence_out), _ptr(commit_out), _ptr(workspace),
                                        ws_bytes, _stream(stream)))


def spork_ngram_workspace_bytes(n_seqs, max_len):
    b = ctypes.c_size_t()
    _check(lib().spork_ngram_workspace_bytes(n_seqs, max_len, ctypes.byref(b)))
    return b.value


def spork_ngram_propose(tokens, seq_off, n_seqs, max_len, n_min, n_max, k, drafts, n_drafts, workspace,
                        stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().spork_ngram_propose(_ptr(tokens), _ptr(seq_off), n_seqs, max_len, n_min, n_max, k,
                                     _ptr(drafts), _ptr(n_drafts), _ptr(workspace), ws_bytes,
                                     _stream(stream)))


# ---- steps whose lengths live on the GPU --------------------------------------
def _bytes(workspace):
    return 0 if workspace is None else workspace.nbytes


def _want(name, x, size, *shape):
    """Device pointer of an integer tensor that the library reads or writes whole, `size` bytes an element (None
    passes: the library says what may be NULL)."""
    if x is None:
        return None
    if x.shape != shape or x.element_size() != size or not x.is_contiguous() or x.is_floating_point() or x.is_complex():
        raise ValueError(f"{name} must be a contiguous tensor of {8 * size}-bit integers of shape {list(shape)}, "
                         f"not {x.dtype} {list(x.shape)}")
    return x.data_ptr()


_element_types = {}
_torch = None


def _of_dtype(dtype, *tensors):
    """Whether all are of the library's dtype, or its bits as integers (integers are pointers and pass)."""
    if not _element_types:
        import torch
        _element_types.update({SPORK_DTYPE_BF16: (torch.bfloat16, torch.int16, torch.uint16),
                               SPORK_DTYPE_F32: (torch.float32, torch.int32, torch.uint32)})
    types = _element_types.get(dtype, ())
    return all(x is None or isinstance(x, int) or x.dtype in types for x in tensors)


def _on_gpu(*tensors):
    """In the memory of the current device, where the launches go (integers are pointers and pass)."""
    here = None
    for x in tensors:
        if x is None or isinstance(x, int):
            continue
        at = x.get_device()
        if at < 0:
            raise ValueError("tensor arguments must be in GPU memory")
        if here is None:
            import torch
            here = torch.cuda.current_device()
        if at != here:
            raise ValueError(f"tensor arguments must be on the current device ({here}), not on {at}")


def make_tables(block_size, table, held, refcount, free_queue, queue):
    """A spork_tables over the given int32 tensors, which it keeps alive: table [n_seqs, max_blocks], held [n_seqs],
    refcount [num_blocks], free_queue [num_blocks], queue [2]."""
    n_seqs, max_blocks = table.shape
    num_blocks = refcount.shape[0]
    t = spork_tables(num_blocks, block_size, n_seqs, max_blocks, _want("table", table, 4, n_seqs, max_blocks),
                     _want("held", held, 4, n_seqs), _want("refcount", refcount, 4, num_blocks),
                     _want("free_queue", free_queue, 4, num_blocks), _want("queue", queue, 4, 2))
    t.tensors = (table, held, refcount, free_queue, queue)
    return t


def spork_tables_init(tables, free_order=None, stream=None):
    order = _want("free_order", free_order, 4, tables.num_blocks)
    _on_gpu(*tables.tensors, free_order)
    _check(lib().spork_tables_init(ctypes.byref(tables), order, _stream(stream)))


def spork_tables_workspace_bytes(tables):
    b = ctypes.c_size_t()
    _check(lib().spork_tables_workspace_bytes(ctypes.byref(tables), ctypes.byref(b)))
    return b.value


def spork_tables_workspace_clear(tables, workspace, stream=None):
    _on_gpu(workspace)
    _check(lib().spork_tables_workspace_clear(ctypes.byref(tables), _ptr(workspace), _bytes(workspace), _stream(stream)))


def spork_tables_step(tables, lens, n_new, parents, slots, positions, row_off, kv_len, copies, n_copies, status,
                      workspace, stream=None):
    """max_tokens is the length of slots."""
    n, most = tables.n_seqs, 0 if slots is None else slots.shape[0]
    args = (_want("lens", lens, 4, n), _want("n_new", n_new, 4, n), _want("parents", parents, 4, n), most,
            _want("slots", slots, 8, most), _want("positions", positions, 4, most), _want("row_off", row_off, 4, n + 1),
            _want("kv_len", kv_len, 4, n), _want("copies", copies, 4, n, 3), _want("n_copies", n_copies, 4, 1),
            _want("status", status, 4, 1), _ptr(workspace), _bytes(workspace))
    _on_gpu(*tables.tensors, lens, n_new, parents, slots, positions, row_off, kv_len, copies, n_copies, status, workspace)
    _check(lib().spork_tables_step(ctypes.byref(tables), *args, _stream(stream)))


def spork_kv_copy_batch(shape, k_cache, v_cache, num_blocks, copies, n_copies, stream=None):
    most = copies.shape[0]
    if not _of_dtype(shape.dtype, k_cache, v_cache):
        raise ValueError("the pools must be of the shape's dtype")
    _on_gpu(k_cache, v_cache, copies, n_copies)
    _check(lib().spork_kv_copy_batch(ctypes.byref(shape), _ptr(k_cache), _ptr(v_cache), num_blocks,
                                     _want("copies", copies, 4, most, 3), _want("n_copies", n_copies, 4, 1),
                                     most, _stream(stream)))


def spork_chunk_workspace_bytes(shape, n_seqs, n_rows):
    b = ctypes.c_size_t()
    _check(lib().spork_chunk_workspace_bytes(ctypes.byref(shape), n_seqs, n_rows, ctypes.byref(b)))
    return b.value


def spork_chunk_attn(shape, q, k_cache, v_cache, table, row_off, kv_len, out, lse, workspace, stream=None):
    """q [rows, hq, head_dim] may have any stride between its rows; num_blocks is the pools' first size."""
    (n_rows, hq, d), (n_seqs, max_blocks), blocks = q.shape, table.shape, k_cache.shape[0]
    if (hq, d) != (shape.hq, shape.head_dim):
        raise ValueError("q must be [rows, hq, head_dim] of the shape")
    if n_rows > 0 and (q.stride(2) != 1 or q.stride(1) != d):
        raise ValueError("the rows of q must be contiguous")
    if tuple(out.shape) != (n_rows, hq, d) or (lse is not None and tuple(lse.shape) != (n_rows, hq)):
        raise ValueError("out must be [rows, hq, head_dim] and lse [rows, hq]")
    if not _of_dtype(shape.dtype, q, k_cache, v_cache, out) or not _of_dtype(SPORK_DTYPE_F32, lse):
        raise ValueError("q, the pools and out must be of the shape's dtype and lse float32")
    bs = shape.block_size
    if tuple(k_cache.shape) != (blocks, shape.hkv, bs, d) or tuple(v_cache.shape) != (blocks, shape.hkv, d, bs):
        raise ValueError("the pools must be [blocks, hkv, block_size, head_dim] and [blocks, hkv, head_dim, block_size]")
    stride = q.stride(0) if n_rows > 1 else hq * d
    args = (q.data_ptr(), stride, _ptr(k_cache), _ptr(v_cache), blocks, _want("table", table, 4, n_seqs, max_blocks),
            max_blocks, _want("row_off", row_off, 4, n_seqs + 1), _want("kv_len", kv_len, 4, n_seqs), n_seqs, n_rows,
            _ptr(out), _ptr(lse), _ptr(workspace), _bytes(workspace))
    _on_gpu(q, k_cache, v_cache, table, row_off, kv_len, out, lse, workspace)
    _check(lib().spork_chunk_attn(ctypes.byref(shape), *args, _stream(stream)))


# ---- from a projection's rows to the cache ------------------------------------------
def spork_rope_frequencies(rotary_dim, base, scaling=None):
    """(float64 array of rotary_dim / 2 frequencies, magnitude); `scaling` is a spork_rope_scaling."""
    freq = np.zeros(max(rotary_dim // 2, 1))
    magnitude = ctypes.c_double()
    _check(lib().spork_rope_frequencies(rotary_dim, float(base), None if scaling is None else ctypes.byref(scaling),
                                        _ptr(freq), ctypes.byref(magnitude)))
    return freq, magnitude.value


def _is_f64(x):
    import torch
    return x.dtype == torch.float64


def make_rope(inv_freq, layout=SPORK_ROPE_HALF, magnitude=1.0):
    """A spork_rope over the float64 tensor inv_freq, two channels a frequency, which it keeps alive."""
    if inv_freq.dim() != 1 or not _is_f64(inv_freq) or not inv_freq.is_contiguous():
        raise ValueError("inv_freq must be a contiguous float64 tensor of one dimension")
    r = spork_rope(2 * inv_freq.shape[0], layout, magnitude, inv_freq.data_ptr())
    r.tensors = (inv_freq,)
    return r


def make_qk_norm(q_weight, k_weight, eps):
    """A spork_qk_norm over weights of head_dim elements (either may be None), which it keeps alive."""
    if any(w is not None and (w.dim() != 1 or not w.is_contiguous()) for w in (q_weight, k_weight)):
        raise ValueError("the norms' weights must be contiguous tensors of one dimension")
    n = spork_qk_norm(_ptr(q_weight), _ptr(k_weight), eps)
    n.tensors = tuple(w for w in (q_weight, k_weight) if w is not None)
    return n


def make_kvq(k_codes, v_codes, k_scale, v_scale):
    """A spork_kvq over tensors of one byte an element (float8_e4m3fn or uint8 codes, uint8 or float8_e8m0fnu scales),
    which it keeps alive: k_codes [blocks, hkv, block_size, head_dim], v_codes [blocks, hkv, head_dim, block_size],
    k_scale and v_scale [blocks, hkv]."""
    import torch
    codes, scales = (torch.float8_e4m3fn, torch.uint8), (torch.uint8, torch.float8_e8m0fnu)
    if k_codes.dim() != 4:
        raise ValueError("k_codes must be [blocks, hkv, block_size, head_dim]")
    blocks, hkv, bs, d = k_codes.shape
    for name, x, shape, types in (("k_codes", k_codes, (blocks, hkv, bs, d), codes), ("v_codes", v_codes, (blocks, hkv, d, bs), codes),
                                  ("k_scale", k_scale, (blocks, hkv), scales), ("v_scale", v_scale, (blocks, hkv), scales)):
        if tuple(x.shape) != shape or x.dtype not in types or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor of {' or '.join(map(str, types))} of shape {list(shape)}, "
                             f"not {x.dtype} {list(x.shape)}")
    c = spork_kvq(blocks, k_codes.data_ptr(), v_codes.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
    c.tensors = (k_codes, v_codes, k_scale, v_scale)
    c.blocks_of = (hkv, bs, d)
    return c


def _types(dtype):
    """The types that tensors of the library's dtype may have, () for one it doesn't know."""
    if not _element_types:
        _of_dtype(dtype)
    return _element_types.get(dtype, ())


def _heads(name, x, shape, types):
    """(device pointer, stride) of rows [n, heads, head_dim] that may have any stride between them; None passes."""
    if x is None:
        return None, 0
    if x.shape != shape or x.dtype not in types:
        raise ValueError(f"{name} must be {list(shape)} of the shape's dtype, not {x.dtype} {list(x.shape)}")
    n, heads, d = shape
    stride = x.stride()
    if n > 0 and (stride[2] != 1 or (stride[1] != d and heads > 1)):
        raise ValueError(f"the rows of {name} must be contiguous")
    return x.data_ptr(), stride[0] if n > 1 else heads * d


def _here(first, *tensors):
    """_on_gpu for tensors alone (None passes, but for the first), without a branch for each kind: the current device."""
    global _torch
    here = first.get_device()
    if here < 0:
        _on_gpu(first)
    if _torch is None:
        import torch
        _torch = torch
    if here != _torch.cuda.current_device():
        _on_gpu(first)
    for x in tensors:
        if x is not None and x.get_device() != here:
            _on_gpu(x)
    return here


def _turn(shape, rope, norm, types):
    """The tensors of rope and norm (None passes)."""
    if norm is None:
        return () if rope is None else rope.tensors
    for w in norm.tensors:
        if w.shape[0] != shape.head_dim or w.dtype not in types:
            raise ValueError("the norms' weights must have head_dim elements of the shape's dtype")
    return norm.tensors if rope is None else rope.tensors + norm.tensors


def spork_qk_rope(shape, rope, norm, positions, q, k, q_out, k_out, stream=None):
    """q [rows, hq, head_dim] and k [rows, hkv, head_dim] (one of them may be None) may have any stride between their
    rows, and so may the outputs; q_out may be q, k_out k."""
    n, d, types = (k if q is None else q).shape[0], shape.head_dim, _types(shape.dtype)
    of_q, of_k = (n, shape.hq, d), (n, shape.hkv, d)
    tensors = _turn(shape, rope, norm, types)
    args = (_want("positions", positions, 4, n), n, *_heads("q", q, of_q, types), *_heads("k", k, of_k, types),
            *_heads("q_out", q_out, of_q, types), *_heads("k_out", k_out, of_k, types))
    here = _here(k if q is None else q, k, q_out, k_out, positions, *tensors)
    _check(lib().spork_qk_rope(ctypes.byref(shape), rope, norm, *args, _stream_at(stream, here)))


def _check_kvq(shape, cache):
    if cache.blocks_of != (shape.hkv, shape.block_size, shape.head_dim):
        raise ValueError("the cache must be of the shape's hkv, block_size and head_dim")


def spork_kvq_write(shape, cache, rope, norm, slots, positions, q, k, v, q_out, bad_slots=None, stream=None):
    """q and q_out [rows, hq, head_dim] (both may be None), k and v [rows, hkv, head_dim] may have any stride between
    their rows; q_out may be q."""
    n, d, types = slots.shape[0], shape.head_dim, _types(shape.dtype)
    of_q, of_k = (n, shape.hq, d), (n, shape.hkv, d)
    _check_kvq(shape, cache)
    tensors = _turn(shape, rope, norm, types)
    args = (_want("slots", slots, 8, n), _want("positions", positions, 4, n), n, *_heads("q", q, of_q, types),
            *_heads("k", k, of_k, types), *_heads("v", v, of_k, types), *_heads("q_out", q_out, of_q, types),
            _want("bad_slots", bad_slots, 4, 1))
    here = _here(*cache.tensors, slots, positions, q, k, v, q_out, bad_slots, *tensors)
    _check(lib().spork_kvq_write(ctypes.byref(shape), cache, rope, norm, *args, _stream_at(stream, here)))


def spork_kvq_copy_batch(shape, cache, copies, n_copies, stream=None):
    most = copies.shape[0]
    _check_kvq(shape, cache)
    args = (_want("copies", copies, 4, most, 3), _want("n_copies", n_copies, 4, 1), most)
    here = _here(*cache.tensors, copies, n_copies)
    _check(lib().spork_kvq_copy_batch(ctypes.byref(shape), cache, *args, _stream_at(stream, here)))


def spork_kvq_attn(shape, q, cache, table, row_off, kv_len, out, lse, workspace, stream=None):
    """q [rows, hq, head_dim] may have any stride between its rows; the workspace is spork_chunk_attn's."""
    n_rows, (n_seqs, max_blocks) = q.shape[0], table.shape
    _check_kvq(shape, cache)
    types, of_q = _types(shape.dtype), (n_rows, shape.hq, shape.head_dim)
    args = (*_heads("q", q, of_q, types), cache, _want("table", table, 4, n_seqs, max_blocks), max_blocks,
            _want("row_off", row_off, 4, n_seqs + 1), _want("kv_len", kv_len, 4, n_seqs), n_seqs, n_rows)
    if out.shape != of_q or out.dtype not in types:
        raise ValueError("out must be [rows, hq, head_dim] of the shape's dtype")
    if lse is not None and (lse.shape != of_q[:2] or lse.dtype not in _types(SPORK_DTYPE_F32)):
        raise ValueError("lse must be [rows, hq] float32")
    here = _here(*cache.tensors, q, table, row_off, kv_len, out, lse, workspace)
    _check(lib().spork_kvq_attn(ctypes.byref(shape), *args, _ptr(out), _ptr(lse), _ptr(workspace), _bytes(workspace),
                                _stream_at(stream, here)))


# ---- measurement aid --------------------------------------------------------
def spork_read_ceiling(src, nbytes, grid, mode, sink, stream=None):
    _check(lib().spork_read_ceiling(_ptr(src), nbytes, grid, mode, _ptr(sink), _stream(stream)))


# ---- kernel timing ------------------------------------------------------------
def spork_timing_enable(on):
    _check(lib().spork_timing_enable(1 if on else 0))


def spork_timing_read():
    """{kernel name: (total ms, launches)} since the last read."""
    ms = np.zeros(SPORK_KERNEL_KINDS, dtype=np.float32)
    n = np.zeros(SPORK_KERNEL_KINDS, dtype=np.int32)
    _check(lib().spork_timing_read(_ptr(ms), _ptr(n)))
    return {KERNEL_NAMES[k]: (float(ms[k]), int(n[k])) for k in range(SPORK_KERNEL_KINDS)}
