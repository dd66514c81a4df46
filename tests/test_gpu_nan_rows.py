"""Query rows that hold a NaN in the planned attention: NaN in their outputs and
lse, and every other row as close to the oracle as without them (twice the parity
tests' tolerance from what it was)."""
import pytest
import torch

from gpu_cases import BF16_TOL, FP32_TOL, LSE_REL, say
from paper_2607_03333_amd import runner, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,make", [
    ("fp32", lambda: synth.make(0)),
    ("4 waves", lambda: synth.make(4, sessions=2, prefix=333, vocab=333)),
    ("8 waves", lambda: synth.make(3, sessions=2, prefix=105, vocab=333, verify_k=23)),
    ("wide", lambda: synth.make(3, sessions=1, prefix=1700, vocab=333, verify_k=24)),
])
def test_a_query_row_that_is_no_number(kernel, make):
    wl = make()
    dw = runner.DeviceWorkload(wl, n_cu=1) if kernel == "wide" else runner.DeviceWorkload(wl)
    try:
        for i in range(len(wl.steps)):
            step = dw.prepare(i)
            step.poison()
            step.run()
            torch.cuda.synchronize()
            out, lse = step.out.clone(), step.lse.clone()
            hit = torch.zeros_like(lse, dtype=torch.bool)
            for row, head in ((0, 0), (lse.shape[0] - 1, lse.shape[1] - 1)):
                hit[row, head] = True
                step.q[row, head, 3] = float("nan")
            step.poison()
            step.run()
            torch.cuda.synchronize()
            assert torch.isnan(step.out[hit]).all() and torch.isnan(step.lse[hit]).all()
            o_rest = (step.out[~hit].float() - out[~hit].float()).abs().max().item()
            l_rest = ((step.lse[~hit] - lse[~hit]).abs() / lse[~hit].abs().clamp(min=1.0)).max().item()
            say(f"  {kernel} step {step.index}: others changed by {o_rest:.2e}, lse {l_rest:.2e}")
            assert o_rest <= 2 * (FP32_TOL if wl.dtype == "f32" else BF16_TOL) and l_rest <= 2 * LSE_REL
    finally:
        dw.close()
