"""norm_fwd with an eps below a float's range, which is not taken for 0."""
import pytest
import torch

from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [1e-300, 1e-50, 1e-46, 1e-45, 1e-38])
def test_rows_without_variance(eps, dtype, gpu):
    """(x - mu) r is 0 for any eps above 0; r is that of the smallest float at most, with a
    rounding each of a root and a reciprocal."""
    want = max(float(torch.tensor(eps)), 2.0 ** -149) ** -0.5
    for d in (5, 1000, 5000):
        for x, rms in ((torch.full((3, d), 2.5), False), (torch.zeros(3, d), True)):
            y, stats = T.norm_fwd(x.to(dtype).cuda(), rms=rms, eps=eps)
            assert not bool(y.any()) and bool(torch.isfinite(stats).all())
            assert bool(((stats[:, 1].double() - want).abs() <= 1e-6 * want).all())
