"""Values of logits that the operators around the logits can go wrong on: largest logits
from a few millions to the edge of fp32, as masks of -1e9, -1e10 or -1e30 on every token of
a row leave them.  Tolerances are those of test_gpu_logprobs.py, whose check is used: the
sums run against a reference that a rounding of up to eight log2 units separates from the
maximum, no more than the eight logits by which it may lag."""
import pytest
import torch

import test_gpu_logprobs as lp

pytestmark = pytest.mark.gpu

LARGEST = [9e6, 6.1e7, 9.9e7, 1.1e8, 1e9, 1.7e9, 1e10, 1.1e10, 7e11, 1e30, 2e30, 7e37, 9.9e37, 3e38]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("n,v,k", [(12, 9001, 5), (800, 9000, 5), (3, 151936, 20), (5, 1000, 7)])
def test_large_logits(n, v, k, sign, dtype, gpu):
    """Rows, in turn: all equal; a peak over ordinary logits (or ordinary logits masked to
    the value in all but a few places); differences of some millionths of the value."""
    for i, m in enumerate(LARGEST):
        m *= sign
        z = lp.normal(n, v, i)
        z[0::3] = m
        if sign > 0:
            z[1::3, v // 3] = m
        else:
            z[1::3, torch.arange(v, device="cuda") % 1000 != 7] = m
        z[2::3] = m + z[2::3].double().mul(abs(m) * 1e-6).clamp(-3e37, 3e37).float()
        lp.check(lp.matrix(n, v, dtype, fill=z), lp.some_ids(n, v, i), k)
