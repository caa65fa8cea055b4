"""Sizes of the workspaces of the operators around the logits (host; no GPU)."""
import itertools

import pytest

from paper_2607_05804_amd import turnkl as T

ROWS = [0, 1, 2, 3, 5, 17, 63, 64, 100, 191, 192, 255, 256, 257, 383, 384, 385, 500, 767, 768, 769, 1000,
        1024, 1279, 1281, 16384, 65536]
VOCABS = [1, 100, 4095, 8191, 8192, 8193, 12288, 32000, 50257, 151936, 196416, 196417, 262144, 400001,
          2 ** 24]


@pytest.mark.parametrize("k", [0, 1, 50, 128])
def test_a_workspace_of_the_largest_call_serves_smaller_ones(k):
    f = T.lib().turnkl_token_logprobs_workspace_bytes
    for v in (v for v in VOCABS if v >= k):
        sizes = [f(n, v, k) for n in ROWS]
        assert sizes == sorted(sizes), (v, k)
        assert all(f(a, v, k) <= f(a + 1, v, k) for a in range(1, 800))
    for n, v in itertools.product(ROWS, (v for v in VOCABS if v >= 128)):
        assert f(n, v, 0) <= f(n, v, 1) <= f(n, v, 50) <= f(n, v, 128)
    for n in ROWS:
        sizes = [f(n, v, k) for v in VOCABS if v >= k]
        assert sizes == sorted(sizes), (n, k)


def test_norm_workspace_does_not_shrink():
    f = T.lib().turnkl_norm_workspace_bytes
    for d in (1, 64, 1000, 2048, 4097, 16384):
        sizes = [f(n, d) for n in range(0, 3000)]
        assert sizes == sorted(sizes), d


def test_only_workspaces_that_hold_a_status_or_segments_are_asked_for_them():
    """A norm's holds sums alone, that of log probabilities no segments."""
    fused = T.Workspace(8, 64, T.F32, 4, device="cpu")
    topk = T.TopkWorkspace(8, 4, 4, device="cpu")
    logprobs = T.LogprobsWorkspace(8, 64, 4, device="cpu")
    norm = T.NormWorkspace(8, 64, device="cpu")
    for ws, status, segments in ((fused, True, True), (topk, True, True), (logprobs, True, False),
                                 (norm, False, False)):
        assert (hasattr(ws, "status"), hasattr(ws, "segments")) == (status, segments), ws
        assert ws.tensor.numel() == ws.nbytes > 0
    for bad in (lambda: T.Workspace(-1, 64, T.F32, 4, device="cpu"), lambda: T.TopkWorkspace(8, 0, 4, device="cpu"),
                lambda: T.LogprobsWorkspace(8, 64, 65, device="cpu"), lambda: T.NormWorkspace(8, 0, device="cpu")):
        with pytest.raises(T.TurnKLError):
            bad()
