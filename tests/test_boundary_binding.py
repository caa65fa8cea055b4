"""The binding of the operators at the token boundary, without a GPU: host tensors and other
types are refused before any address reaches the library; with a library that only records,
every call goes to its tensors' device and stream."""
import pytest
import torch

from paper_2607_05804_amd import turnkl as T
from test_operator_devices import STREAMS, THERE, library  # noqa: F401

X = torch.zeros(4, 16)
B = X.bfloat16()
W = torch.zeros(16)
U = torch.zeros(4, dtype=torch.float64)
ID = torch.zeros(4, dtype=torch.int32)
STATS = torch.zeros(4, 2)

CALLS = [
    ("turnkl_sample_tokens", lambda: T.sample_tokens(X, U, check=False)),
    ("turnkl_sample_tokens", lambda: T.sample_tokens(B, U, temperature=torch.ones(4), top_k=ID, check=False)),
    ("turnkl_embed_fwd", lambda: T.embed_fwd(X, ID, dtype=torch.bfloat16)),
    ("turnkl_embed_bwd", lambda: T.embed_bwd(B, ID, X, check=False)),
    ("turnkl_block_norm_fwd", lambda: T.block_norm_fwd(X, B, W, gate=W)),
    ("turnkl_block_norm_bwd", lambda: T.block_norm_bwd(B, X, X, STATS, B, W, gate=B)),
]


@pytest.mark.parametrize("name,call", CALLS)
def test_host_tensors_are_refused(name, call):
    with pytest.raises(ValueError, match="on the GPU"):
        call()


@pytest.mark.parametrize("name,call", CALLS)
def test_calls_go_to_the_tensors_device(name, call, library):  # noqa: F811
    call()
    assert library.calls == [(name, THERE, [STREAMS[THERE]])]


@pytest.mark.parametrize("name,call", [
    ("turnkl_sample_tokens", lambda: T.sample_tokens(X, U)), ("turnkl_embed_bwd", lambda: T.embed_bwd(X, ID, X.clone()))])
def test_the_status_is_read_where_the_call_went(name, call, library):  # noqa: F811
    call()
    assert library.calls == [(name, THERE, [STREAMS[THERE]]), ("turnkl_get_status", THERE, [STREAMS[THERE]])]


def test_other_types_are_refused(library):  # noqa: F811
    for call in (lambda: T.sample_tokens(X.half(), U), lambda: T.embed_fwd(X.double(), ID),
                 lambda: T.embed_bwd(X, ID, X.half()), lambda: T.block_norm_fwd(X.double(), X)):
        with pytest.raises(TypeError):
            call()


def test_which_workspaces_hold_a_status():
    for ws, status in ((T.SampleWorkspace(8, 64, device="cpu"), True), (T.EmbedWorkspace(8, 64, 32, device="cpu"), True),
                       (T.BlockNormWorkspace(8, 64, device="cpu"), False)):
        assert hasattr(ws, "status") == status and ws.tensor.numel() == ws.nbytes > 0
    for bad in (lambda: T.SampleWorkspace(8, 0, device="cpu"), lambda: T.EmbedWorkspace(8, 64, 0, device="cpu"),
                lambda: T.BlockNormWorkspace(-1, 64, device="cpu")):
        with pytest.raises(T.TurnKLError):
            bad()


def test_buffers_for_gradients():
    g = T.new_block_norm_grads(3, 8, torch.bfloat16, torch.float32, gate="matrix", post_weight=True, pad_cols=2,
                               device="cpu")
    assert g.residual.dtype == torch.float32 and g.branch.stride(0) == 10 and g.gate.dtype == torch.bfloat16
    assert g.bias is None and g.weight.shape == g.post_weight.shape == (8,)
    assert T.new_block_norm_grads(3, 8, gate="vector", weight=False, device="cpu").gate.shape == (8,)
    with pytest.raises(ValueError):
        T.new_block_norm_grads(3, 8, gate="scalar", device="cpu")


@pytest.mark.parametrize("given,passed", [(0, 0), (7, 7), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1),
                                          (-2 ** 40, -2 ** 31)])
def test_top_k_does_not_wrap(given, passed, library, monkeypatch):  # noqa: F811
    seen = []

    def call(*a):
        seen.extend(x.top_k for x in a if isinstance(x, T.Sampling))
        return T.OK

    library.turnkl_sample_tokens = call
    T.sample_tokens(X, U, top_k=given, check=False)
    assert seen == [passed]
    with pytest.raises(TypeError):
        T.sample_tokens(X, U, top_k=2.5, check=False)
