"""What the binding of the operators around the logits hands to the library for buffers
whose rows lie in an unusual way, with host tensors and a library that only records (the
device checks are taken out; no address is read)."""
import pytest
import torch

from paper_2607_05804_amd import turnkl as T


class Recorder:
    """Stands for the library: records the log probabilities' row stride of alternatives
    and refuses one below k, as turnkl.h says."""

    def turnkl_token_logprobs_workspace_bytes(self, n, v, k):
        return 256

    def turnkl_token_logprobs(self, *a):
        self.n, self.k, self.ld_top = a[3], a[7], a[13]
        return T.ERR_INVALID_ARG if self.n > 0 and self.ld_top < self.k else T.OK


@pytest.fixture
def library(monkeypatch):
    stub, real = Recorder(), T.lib()
    monkeypatch.setattr(T, "lib", lambda: stub)
    monkeypatch.setattr(T, "_gpu", lambda t: t.get_device())
    monkeypatch.setattr(T, "_stream", lambda index: 0)
    monkeypatch.setattr(T, "_on", lambda index, call: call)
    monkeypatch.setattr(T, "status_string", lambda code: real.turnkl_status_string(code).decode())
    return stub


def alternatives(n, k, ids, logp):
    return T.TokenLogprobs(None, torch.empty(n), torch.empty(n, 2), ids, logp)


def call(out, n, k):
    return T.token_logprobs(torch.zeros(n, 64), k=k, out=out, check=False)


@pytest.mark.parametrize("n,k", [(2, 3), (5, 7)])
def test_rows_of_alternatives_that_overlap_are_refused(n, k, library):
    """Their storage is smaller than n rows of k."""
    whole = torch.empty(n, k)
    for make in (lambda d: torch.empty((1, k), dtype=d).expand(n, k),
                 lambda d: torch.empty(n * k, dtype=d).as_strided((n, k), (1, 1)),
                 lambda d: torch.empty(n * k, dtype=d).as_strided((n, k), (k - 1, 1))):
        with pytest.raises(T.TurnKLError) as e:
            call(alternatives(n, k, make(torch.int32), make(torch.float32)), n, k)
        assert e.value.code == T.ERR_INVALID_ARG
        with pytest.raises((T.TurnKLError, ValueError)):
            call(alternatives(n, k, whole.int(), make(torch.float32)), n, k)


@pytest.mark.parametrize("n,k,ld", [(4, 3, 3), (4, 3, 8), (1, 3, 8), (0, 3, 3)])
def test_strides_of_alternatives(n, k, ld, library):
    ids, logp = (torch.empty((n, ld), dtype=d)[:, :k] for d in (torch.int32, torch.float32))
    call(alternatives(n, k, ids, logp), n, k)
    assert library.n == n and library.ld_top >= k and (n < 2 or library.ld_top == ld)


def test_a_single_row_of_alternatives_has_no_stride_to_share(library):
    """One row may lie in two buffers of their own widths; rows at two strides may not."""
    ids, logp = torch.empty((1, 9), dtype=torch.int32)[:, :3], torch.empty((1, 3))
    call(alternatives(1, 3, ids, logp), 1, 3)
    assert library.ld_top >= 3
    ids, logp = torch.empty((2, 9), dtype=torch.int32)[:, :3], torch.empty((2, 3))
    with pytest.raises(ValueError, match="share a row stride"):
        call(alternatives(2, 3, ids, logp), 2, 3)
