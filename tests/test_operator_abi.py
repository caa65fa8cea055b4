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


def logprobs_bwd(**kw):
    n, v = kw.get("n", 64), kw.get("v", 1024)
    a = dict(z=0x100000000, ld=v, dtype=T.BF16, n=n, v=v, ids=0x200000000, mask=0x210000000,
             lz=0x220000000, h=0x230000000, gl=0x240000000, gh=0x250000000, grad=0x300000000, ld_g=v)
    a.update(kw)
    return T.lib().turnkl_token_logprobs_bwd(
        P(a["z"]), a["ld"], a["dtype"], a["n"], a["v"], P(a["ids"]), P(a["mask"]), P(a["lz"]), P(a["h"]),
        P(a["gl"]), P(a["gh"]), P(a["grad"]), a["ld_g"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), T.ERR_INVALID_ARG),
    (dict(n=-1), T.ERR_INVALID_ARG),
    (dict(v=0), T.ERR_INVALID_ARG),
    (dict(v=2 ** 24 + 1), T.ERR_INVALID_ARG),
    (dict(z=0), T.ERR_INVALID_ARG),
    (dict(lz=0), T.ERR_INVALID_ARG),
    (dict(grad=0), T.ERR_INVALID_ARG),
    (dict(gl=0, gh=0), T.ERR_INVALID_ARG),
    (dict(ids=0), T.ERR_INVALID_ARG),
    (dict(h=0), T.ERR_INVALID_ARG),
    (dict(ld=1000), T.ERR_INVALID_ARG),
    (dict(ld_g=1000), T.ERR_INVALID_ARG),
    (dict(ld_g=2 ** 31), T.ERR_INVALID_ARG),
    (dict(grad=0x300000001), T.ERR_INVALID_ARG),
    (dict(gh=0x250000003), T.ERR_INVALID_ARG),
    (dict(grad=0x100000002), T.ERR_ALIAS),
    (dict(grad=0x100000000, ld_g=2048), T.ERR_ALIAS),
    (dict(grad=0x220000000 - 64 * 2048 + 4), T.ERR_ALIAS),
    (dict(grad=0x250000000), T.ERR_ALIAS),
    (dict(grad=0x210000000), T.ERR_ALIAS),
    (dict(n=0, z=0, lz=0, grad=0), T.OK),
])
def test_logprobs_bwd_refuses(kw, code):
    assert logprobs_bwd(**kw) == code


def norm_fwd(**kw):
    n, d = kw.get("n", 64), kw.get("d", 1024)
    a = dict(x=0x100000000, ld_x=d, dtype=T.BF16, n=n, d=d, w=0x200000000, b=0x210000000, pt=T.BF16,
             kind=T.NORM_LAYER, eps=1e-6, y=0x300000000, ld_y=d, st=0x220000000)
    a.update(kw)
    return T.lib().turnkl_norm_fwd(P(a["x"]), a["ld_x"], a["dtype"], a["n"], a["d"], P(a["w"]), P(a["b"]),
                                   a["pt"], a["kind"], a["eps"], P(a["y"]), a["ld_y"], P(a["st"]), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), T.ERR_INVALID_ARG),
    (dict(pt=3), T.ERR_INVALID_ARG),
    (dict(kind=2), T.ERR_INVALID_ARG),
    (dict(n=-1), T.ERR_INVALID_ARG),
    (dict(n=2 ** 31), T.ERR_INVALID_ARG),
    (dict(d=0), T.ERR_INVALID_ARG),
    (dict(d=16385), T.ERR_INVALID_ARG),
    (dict(d=2 ** 62), T.ERR_INVALID_ARG),
    (dict(eps=-1e-9), T.ERR_INVALID_ARG),
    (dict(eps=float("nan")), T.ERR_INVALID_ARG),
    (dict(eps=float("inf")), T.ERR_INVALID_ARG),
    (dict(x=0), T.ERR_INVALID_ARG),
    (dict(y=0), T.ERR_INVALID_ARG),
    (dict(ld_x=1023), T.ERR_INVALID_ARG),
    (dict(ld_y=1023), T.ERR_INVALID_ARG),
    (dict(x=0x100000001), T.ERR_INVALID_ARG),
    (dict(w=0x200000001), T.ERR_INVALID_ARG),
    (dict(b=0x210000002, pt=T.F32), T.ERR_INVALID_ARG),
    (dict(st=0x220000002), T.ERR_INVALID_ARG),
    (dict(y=0x100000010), T.ERR_ALIAS),
    (dict(y=0x100000000, ld_y=1032), T.ERR_ALIAS),
    (dict(y=0x200000000), T.ERR_ALIAS),
    (dict(st=0x300000000 + 64), T.ERR_ALIAS),
    (dict(st=0x100000000), T.ERR_ALIAS),
    (dict(n=0, x=0, y=0), T.OK),
])
def test_norm_fwd_refuses(kw, code):
    assert norm_fwd(**kw) == code


def norm_bwd(**kw):
    n, d = kw.get("n", 64), kw.get("d", 1024)
    a = dict(g=0x100000000, ld_g=d, x=0x110000000, ld_x=d, dtype=T.BF16, n=n, d=d, w=0x200000000,
             pt=T.BF16, kind=T.NORM_LAYER, st=0x210000000, gx=0x300000000, ld_gx=d, gw=0x310000000,
             gb=0x320000000, acc=0, ws=0x400000000, wb=T.lib().turnkl_norm_workspace_bytes(n, d))
    a.update(kw)
    return T.lib().turnkl_norm_bwd(P(a["g"]), a["ld_g"], P(a["x"]), a["ld_x"], a["dtype"], a["n"], a["d"],
                                   P(a["w"]), a["pt"], a["kind"], P(a["st"]), P(a["gx"]), a["ld_gx"],
                                   P(a["gw"]), P(a["gb"]), a["acc"], P(a["ws"]), a["wb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), T.ERR_INVALID_ARG),
    (dict(kind=-1), T.ERR_INVALID_ARG),
    (dict(d=16385), T.ERR_INVALID_ARG),
    (dict(gx=0, gw=0, gb=0), T.ERR_INVALID_ARG),
    (dict(g=0), T.ERR_INVALID_ARG),
    (dict(x=0), T.ERR_INVALID_ARG),
    (dict(st=0), T.ERR_INVALID_ARG),
    (dict(ld_g=1023), T.ERR_INVALID_ARG),
    (dict(ld_gx=1023), T.ERR_INVALID_ARG),
    (dict(gw=0x310000001), T.ERR_INVALID_ARG),
    (dict(ws=0), T.ERR_INVALID_ARG),
    (dict(ws=0x400000010), T.ERR_WORKSPACE),
    (dict(wb=1024), T.ERR_WORKSPACE),
    (dict(gx=0x100000002), T.ERR_ALIAS),
    (dict(gx=0x110000000, ld_gx=2048), T.ERR_ALIAS),
    (dict(gx=0x100000000, x=0x100000000 + 64), T.ERR_ALIAS),
    (dict(gw=0x320000000 + 16), T.ERR_ALIAS),
    (dict(gw=0x110000000 + 16), T.ERR_ALIAS),
    (dict(gb=0x210000000), T.ERR_ALIAS),
    (dict(gb=0x300000000 + 64), T.ERR_ALIAS),
    (dict(ws=0x300000000), T.ERR_ALIAS),
    (dict(ws=0x200000000), T.ERR_ALIAS),
])
def test_norm_bwd_refuses(kw, code):
    assert norm_bwd(**kw) == code


def test_norm_workspace():
    f = T.lib().turnkl_norm_workspace_bytes
    assert f(-1, 10) == 0 and f(10, 0) == 0 and f(10, 16385) == 0 and f(2 ** 31, 10) == 0
    assert 0 < f(0, 10) <= f(10, 10) < f(10 ** 6, 10) < f(10 ** 6, 16384)
    assert f(10 ** 6, 4096) % 256 == 0
