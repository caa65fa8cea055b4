"""One workspace of token log probabilities for batches of every size up to its own."""
import pytest
import torch

import test_gpu_logprobs as lp
from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_most,v,k", [(2000, 20001, 50), (800, 151936, 128), (5, 400001, 20)])
def test_smaller_calls_share_the_largest_ones_workspace(n_most, v, k, gpu):
    ws = T.LogprobsWorkspace(n_most, v, k)
    for n, cols, alternatives in ((n_most, v, k), (1, v, k), (3, v, k), (min(n_most, 64), v, k),
                                  (min(n_most, 384), v, 1), (2, 9001, k), (1, 300, 7)):
        ws.tensor.fill_(0xA5)
        z = lp.matrix(n, cols, "bf16", fill=lp.normal(n, cols, n))
        lp.check(z, lp.some_ids(n, cols, n), alternatives, workspace=ws)


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 4])
def test_as_many_rows_as_are_admitted(n, gpu):
    """Rows of one column, of which the last four are asked for: log p of the only token
    is 0, and the others' outputs are those of rows that are not."""
    z = torch.zeros((n, 1), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    z[:-4] = float("nan")
    mask[-4:] = 1
    log_z = torch.full((n, 2), 7.0, device="cuda")
    out = T.TokenLogprobs(torch.full((n,), 7.0, device="cuda"), None, log_z, None, None)
    T.token_logprobs(z, ids, mask=mask, out=out)
    for part in out.logp.split(1 << 28):
        assert not bool(part.any())
    assert bool((log_z[-4:] == 0).all())
    for part in log_z[:-4].split(1 << 28):
        assert bool(part.isnan().all())
