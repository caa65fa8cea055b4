"""Every call of the binding reaches the library with the tensors' device current and with
that device's stream, whichever device is current for the caller: the default stream's
address is 0 on all of them.  Host tensors (device -1) stand for those of another GPU, and
a library that only records for the real one."""
import pytest
import torch

from paper_2607_05804_amd import turnkl as T

HERE, THERE = 0, -1  # the caller's device, the tensors'


class Recorder:
    def __init__(self, device):
        self.device, self.calls = device, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 256

        def call(*a):
            self.calls.append((name, self.device[0], [x for x in a if x in STREAMS.values()]))
            return T.OK

        return call


STREAMS = {HERE: 0x1111, THERE: 0x2222}


@pytest.fixture
def library(monkeypatch):
    current = [HERE]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *a):
            current[0] = self.before

    class Stream:
        def __init__(self, device=None):
            at = current[0] if device is None else THERE
            self.cuda_stream = STREAMS[at]

    stub = Recorder(current)
    monkeypatch.setattr(T, "lib", lambda: stub)
    monkeypatch.setattr(T, "_gpu", lambda t: t.get_device())
    monkeypatch.setattr(T, "_current_device", lambda: current[0])
    monkeypatch.setattr(T, "_stream", lambda index: STREAMS[index])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(T.ctypes, "c_void_p", lambda x: x)
    monkeypatch.setattr(T.ctypes, "byref", lambda x: None)
    yield stub
    assert current[0] == HERE


X = torch.zeros(4, 16)
VEC = torch.zeros(4)
ID = torch.zeros(4, dtype=torch.int32)
ON = torch.ones(4, dtype=torch.uint8)
STATS = torch.zeros(4, 2)


@pytest.mark.parametrize("name,call", [
    ("turnkl_token_logprobs", lambda: T.token_logprobs(X, ID, k=2, check=False)),
    ("turnkl_token_logprobs_bwd", lambda: T.token_logprobs_bwd(X, ID, STATS, VEC, grad_logp=VEC)),
    ("turnkl_norm_fwd", lambda: T.norm_fwd(X)),
    ("turnkl_norm_bwd", lambda: T.norm_bwd(X, X, None, STATS)),
    ("turnkl_fwd_bwd", lambda: T.fwd_bwd(X, X, ID, ID, ON, 0.5, check=False)),
    ("turnkl_fwd_bwd_noalloc", lambda: T.fwd_bwd_noalloc(X, X, ID, ID, ON, 0.5, torch.zeros(3))),
    ("turnkl_fwd_bwd_topk", lambda: T.fwd_bwd_topk(X, ID.view(4, 1), X[:, :1].clone(), ID, ID, ON, 0.5,
                                                   check=False)),
    ("turnkl_get_status", lambda: T.LogprobsWorkspace(4, 16, device="cpu").status()),
    ("turnkl_get_status", lambda: T.Workspace(4, 16, T.F32, 2, device="cpu").status()),
    ("turnkl_get_segments", lambda: T.Workspace(4, 16, T.F32, 2, device="cpu").segments()),
])
def test_calls_go_to_the_tensors_device(name, call, library):
    call()
    assert library.calls == [(name, THERE, [STREAMS[THERE]])]


def test_the_status_is_read_where_the_call_went(library):
    T.token_logprobs(X, ID)
    assert library.calls == [("turnkl_token_logprobs", THERE, [STREAMS[THERE]]),
                             ("turnkl_get_status", THERE, [STREAMS[THERE]])]
