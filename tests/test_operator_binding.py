"""The binding of the operators around the logits refuses tensors that are not on the
GPU, before any address reaches the library."""
import pytest
import torch

from paper_2607_05804_amd import turnkl as T

X = torch.zeros(3, 8)
STATS = torch.zeros(3, 2)


@pytest.mark.parametrize("call", [
    lambda: T.token_logprobs(X), lambda: T.token_logprobs(X.bfloat16(), k=2),
    lambda: T.token_logprobs_bwd(X, None, STATS, X[:, 0], grad_entropy=X[:, 0]),
    lambda: T.norm_fwd(X), lambda: T.norm_bwd(X, X, None, STATS)])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError, match="on the GPU"):
        call()


def test_types_are_refused_before_that():
    for call in (lambda: T.token_logprobs(X.half()), lambda: T.norm_fwd(X.double())):
        with pytest.raises(TypeError):
            call()
