"""What the binding keeps of a projection's rows and of the cache of 8-bit codes, on
the CPU: a rope, norm or cache keeps its tensors alive as long as it lives itself, and
no longer."""
import ctypes
import gc
import weakref

import pytest

from paper_2607_03333_amd import spork

torch = pytest.importorskip("torch")


def _pools(blocks=3, hkv=2, bs=16, d=64):
    u8 = lambda *m: torch.zeros(m, dtype=torch.uint8)  # noqa: E731
    return [u8(blocks, hkv, bs, d), u8(blocks, hkv, d, bs), u8(blocks, hkv), u8(blocks, hkv)]


MAKERS = [(spork.make_rope, lambda: [torch.zeros(32, dtype=torch.float64)], ()),
          (spork.make_qk_norm, lambda: [torch.ones(64), torch.ones(64)], (1e-6,)),
          (spork.make_kvq, _pools, ())]


@pytest.mark.parametrize("used", (False, True))
@pytest.mark.parametrize("make,tensors,more", MAKERS)
def test_tensors_live_as_long_as_what_is_made_of_them(make, tensors, more, used):
    held = tensors()
    alive = [weakref.ref(x) for x in held]
    made = make(*held, *more)
    del held
    gc.collect()
    assert all(x() is not None for x in alive)
    if used:
        _pass_through(made)
    del made
    gc.collect()
    assert not any(x() is not None for x in alive)


def _pass_through(made):
    """Every call that takes it, with nothing to do or refused for tensors that aren't on the GPU."""
    shape = spork.make_shape(4, 2, 64, 16, spork.SPORK_DTYPE_F32, 0.1)
    rope = made if isinstance(made, spork.spork_rope) else None
    norm = made if isinstance(made, spork.spork_qk_norm) else None if rope else spork.make_qk_norm(torch.ones(64), torch.ones(64), 0.0)
    cache = made if isinstance(made, spork.spork_kvq) else spork.make_kvq(*_pools())
    i32 = lambda *m: torch.zeros(m, dtype=torch.int32)  # noqa: E731
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    for call in (lambda: spork.spork_qk_rope(shape, rope, norm, i32(3), q, k, q, k),
                 lambda: spork.spork_kvq_write(shape, cache, rope, norm, i32(3).long(), i32(3), q, k, k.clone(), q),
                 lambda: spork.spork_kvq_copy_batch(shape, cache, i32(2, 3), i32(1)),
                 lambda: spork.spork_kvq_attn(shape, q, cache, i32(2, 4), i32(3), i32(2), q.clone(), None, torch.zeros(64))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    lib = spork.lib()
    refs = (ctypes.byref(shape), rope, norm)
    assert lib.spork_qk_rope(*refs, None, 0, *[None, 0] * 4, None) == 0
    assert lib.spork_kvq_write(refs[0], cache, *refs[1:], None, None, 0, *[None, 0] * 4, None, None) == 0
    assert lib.spork_kvq_copy_batch(refs[0], cache, None, None, 0, None) == 0
