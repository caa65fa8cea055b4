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
