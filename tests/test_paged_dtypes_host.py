"""The binding of the steps whose lengths live on the GPU takes tensors of the
shape's type (or its bits as integers) and no others of the same width. On the CPU:
what passes that check is then refused for its place."""
import pytest
import torch

from paper_2607_03333_amd import spork

pytestmark = pytest.mark.filterwarnings("ignore:ComplexHalf")
BF16, F32 = spork.SPORK_DTYPE_BF16, spork.SPORK_DTYPE_F32
RIGHT = {BF16: (torch.bfloat16, torch.int16), F32: (torch.float32, torch.int32)}
WRONG = {BF16: (torch.float16, torch.float32, torch.int32), F32: (torch.bfloat16, torch.float64, torch.int64, torch.complex32)}


def i32(*m):
    return torch.zeros(m, dtype=torch.int32)


def attention(code, dtype, which=None, other=None):
    types = dict(q=dtype, k=dtype, v=dtype, out=dtype, lse=torch.float32)
    if which:
        types[which] = other
    sizes = dict(q=(3, 4, 64), k=(5, 2, 16, 64), v=(5, 2, 64, 16), out=(3, 4, 64), lse=(3, 4))
    t = {name: torch.empty(size, dtype=types[name]) for name, size in sizes.items()}
    spork.spork_chunk_attn(spork.make_shape(4, 2, 64, 16, code, 0.1), t["q"], t["k"], t["v"], i32(2, 4), i32(3), i32(2), t["out"],
                           t["lse"], torch.zeros(64), stream=0)


@pytest.mark.parametrize("code", (BF16, F32))
def test_attention_takes_the_shapes_type(code):
    for dtype in RIGHT[code]:
        with pytest.raises(ValueError, match="GPU memory"):
            attention(code, dtype)
    for which in ("q", "k", "v", "out"):
        for other in WRONG[code]:
            with pytest.raises(ValueError, match="dtype"):
                attention(code, RIGHT[code][0], which, other)
    for other in (torch.float16, torch.float64, torch.bfloat16, torch.complex32):
        with pytest.raises(ValueError, match="lse float32"):
            attention(code, RIGHT[code][0], "lse", other)


@pytest.mark.parametrize("code", (BF16, F32))
def test_copies_take_the_shapes_type(code):
    shape = spork.make_shape(4, 2, 64, 16, code, 0.1)

    def copy(k, v):
        spork.spork_kv_copy_batch(shape, torch.empty(5, 2, 16, 64, dtype=k), torch.empty(5, 2, 64, 16, dtype=v), 5, i32(2, 3), i32(1),
                                  stream=0)

    right = RIGHT[code][0]
    for dtype in RIGHT[code]:
        with pytest.raises(ValueError, match="GPU memory"):
            copy(dtype, dtype)
    for other in WRONG[code]:
        for pair in ((right, other), (other, right)):
            with pytest.raises(ValueError, match="dtype"):
                copy(*pair)


def test_integers_are_integers():
    t = spork.make_tables(16, i32(2, 4), i32(2), i32(9), i32(9), i32(2))
    for slots in (torch.empty(5, dtype=torch.complex64), torch.empty(5, dtype=torch.float64)):
        with pytest.raises(ValueError, match="slots"):
            spork.spork_tables_step(t, i32(2), i32(2), None, slots, i32(5), i32(3), i32(2), i32(2, 3), i32(1), i32(1),
                                    torch.zeros(1 << 12, dtype=torch.uint8), stream=0)
