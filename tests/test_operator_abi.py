"""Host-side checks of the operators around the logits: every call here returns
before the first HIP runtime call (no GPU needed; addresses are never read)."""
import ctypes

import pytest

from paper_2607_05804_amd import turnkl as T

P = lambda x: ctypes.c_void_p(x) if x else None  # noqa: E731


def logprobs(**kw):
    n, v, k = kw.get("n", 64), kw.get("v", 1024), kw.get("k", 8)
    a = dict(z=0x100000000, ld=v, dtype=T.BF16, n=n, v=v, ids=0x200000000, mask=0x210000000, k=k,
             logp=0x220000000, h=0x230000000, lz=0x240000000, ti=0x250000000, tp=0x260000000,
             ld_top=k, ws=0x500000000,
             ws_bytes=T.lib().turnkl_token_logprobs_workspace_bytes(n, v, k))
    a.update(kw)
    return T.lib().turnkl_token_logprobs(
        P(a["z"]), a["ld"], a["dtype"], a["n"], a["v"], P(a["ids"]), P(a["mask"]), a["k"],
        P(a["logp"]), P(a["h"]), P(a["lz"]), P(a["ti"]), P(a["tp"]), a["ld_top"], P(a["ws"]),
        a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), T.ERR_INVALID_ARG),
    (dict(n=-1), T.ERR_INVALID_ARG),
    (dict(n=2 ** 31), T.ERR_INVALID_ARG),
    (dict(v=0), T.ERR_INVALID_ARG),
    (dict(v=2 ** 24 + 1), T.ERR_INVALID_ARG),
    (dict(k=-1), T.ERR_INVALID_ARG),
    (dict(k=129), T.ERR_INVALID_ARG),
    (dict(k=9, v=8), T.ERR_INVALID_ARG),
    (dict(z=0), T.ERR_INVALID_ARG),
    (dict(z=0x100000001), T.ERR_INVALID_ARG),
    (dict(z=0x100000002, dtype=T.F32), T.ERR_INVALID_ARG),
    (dict(ld=1023), T.ERR_INVALID_ARG),
    (dict(ld=2 ** 31), T.ERR_INVALID_ARG),
    (dict(ids=0), T.ERR_INVALID_ARG),  # log probabilities of no tokens
    (dict(ids=0x200000002), T.ERR_INVALID_ARG),
    (dict(logp=0x220000001), T.ERR_INVALID_ARG),
    (dict(lz=0x240000002), T.ERR_INVALID_ARG),
    (dict(ti=0), T.ERR_INVALID_ARG),
    (dict(tp=0), T.ERR_INVALID_ARG),
    (dict(ld_top=7), T.ERR_INVALID_ARG),
    (dict(k=0), T.ERR_INVALID_ARG),  # alternatives' buffers without alternatives
    (dict(ws=0), T.ERR_INVALID_ARG),
    (dict(ws=0x500000080), T.ERR_WORKSPACE),
    (dict(ws_bytes=255), T.ERR_WORKSPACE),
    (dict(logp=0x100000000 + 64), T.ERR_ALIAS),
    (dict(h=0x200000000 + 252), T.ERR_ALIAS),
    (dict(lz=0x210000000 + 60), T.ERR_ALIAS),
    (dict(lz=0x220000000 - 8), T.ERR_ALIAS),
    (dict(ti=0x260000000 + 4), T.ERR_ALIAS),
    (dict(h=0x500000000), T.ERR_ALIAS),
    (dict(ws=0x100000000), T.ERR_ALIAS),
])
def test_logprobs_refuses(kw, code):
    assert logprobs(**kw) == code


def test_logprobs_workspace():
    f = T.lib().turnkl_token_logprobs_workspace_bytes
    assert f(-1, 100, 0) == 0 and f(10, 0, 0) == 0 and f(10, 2 ** 24 + 1, 0) == 0
    assert f(10, 100, 129) == 0 and f(10, 100, -1) == 0 and f(10, 5, 6) == 0
    assert f(0, 100, 0) >= 256
    assert f(10, 2 ** 24, 128) > f(10, 2 ** 24, 1) > f(10, 2 ** 24, 0) > f(10, 1000, 0)
    assert f(65536, 151936, 50) < 16 << 20  # a batch that fills the card needs no room for chunks


def test_status_string():
    assert "token" in T.status_string(T.ERR_TOKEN_ID)
