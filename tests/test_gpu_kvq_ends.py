"""The largest numbers on their way through the cache of 8-bit codes
(spork_kvq_write, spork_kvq_attn): a value comes back as its nearest code times the
scale as long as that is below 2^128, and as an infinity from there on, which
spoils its own channel and no other."""
import numpy as np
import pytest
import torch

from paper_2607_03333_amd import spork
from rows_cases import PoolModel
from test_gpu_rope import BF16, F32, SPORK

pytestmark = pytest.mark.gpu

EDGE = 248 * 2.0 ** 120  # half way from the code 240 to 256, which times 2^120 is 2^128


@pytest.mark.parametrize("rows", (1, 20))
@pytest.mark.parametrize("dtype,d,bs", [(BF16, 64, 16), (BF16, 128, 32), (F32, 64, 32), (F32, 128, 16)])
def test_values_up_to_the_largest_number(dtype, d, bs, rows):
    """`rows` new tokens of a sequence whose first token's values are the largest ones; the others' weigh nothing beside it."""
    hq, hkv = 8, 2
    rng = np.random.default_rng(d + bs)
    values = [3.3e38, -3.3e38, 3.38e38, EDGE, -EDGE, float(np.nextafter(np.float32(EDGE), np.float32(0))), 3.2e38, -3.2e38, 240 * 2.0 ** 120,
              2.0 ** 127, 1.7e38]
    v = torch.zeros(rows, hkv, d, dtype=dtype)
    v[0, 1, :len(values)] = torch.tensor(values, dtype=torch.float64).to(torch.float32).to(dtype)
    v[0, 0] = torch.from_numpy(rng.standard_normal(d)).to(dtype)
    k = torch.zeros(rows, hkv, d, dtype=dtype)
    k[0] = 1.0
    q = torch.full((rows, hq, d), 64.0, dtype=dtype).cuda()  # scores of 64 sqrt(d), and of zero
    blocks = -(-rows // bs)
    u8 = lambda *m: torch.zeros(m, dtype=torch.uint8, device="cuda")  # noqa: E731
    pools = [u8(blocks, hkv, bs, d), u8(blocks, hkv, d, bs), u8(blocks, hkv), u8(blocks, hkv)]
    cache, shape = spork.make_kvq(*pools), spork.make_shape(hq, hkv, d, bs, SPORK[dtype], d ** -0.5)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    spork.spork_kvq_write(shape, cache, None, None, torch.arange(rows, device="cuda"), None, None, k.cuda(), v.cuda(), None)
    out, lse = torch.zeros(rows, hq, d, dtype=dtype, device="cuda"), torch.zeros(rows, hq, device="cuda")
    ws = torch.zeros(spork.spork_chunk_workspace_bytes(shape, 1, rows), dtype=torch.uint8, device="cuda")
    spork.spork_kvq_attn(shape, q, cache, i32(*range(blocks)).view(1, blocks), i32(0, rows), i32(rows), out, lse, ws)
    torch.cuda.synchronize()
    model = PoolModel(np.zeros((blocks, hkv, bs, d), np.uint8), np.full((blocks, hkv), 127))
    for b in range(blocks):
        model.write(b, 0, v[b * bs:(b + 1) * bs].double().numpy())
    held = torch.from_numpy(model.values(0, 1)[0])  # [hkv][d] in float64: 2^128 among them
    past = held.abs() >= 2.0 ** 128
    assert past[1, :5].tolist() == [float(x) != 0 and abs(float(x)) >= EDGE for x in v[0, 1, :5].double()] and past[1, 0]
    assert not past[1, 6:9].any()
    want = torch.where(past, torch.sign(held) * float("inf"), held).to(torch.float32).to(dtype).repeat_interleave(hq // hkv, 0)
    got = out.cpu()
    assert torch.isfinite(lse).all()
    # the probability of the first token is 1, those of the others are zero in 32 bits: outputs are the values
    for r in range(rows):
        assert torch.equal(got[r], want), r
