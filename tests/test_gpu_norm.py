"""turnkl_norm_fwd and turnkl_norm_bwd against their formulas in 64 bits and against
central differences.

Tolerances (u = 2^-24).  Sums of a row: at most 32 terms in sequence per thread and
a tree of 20, so 60 u of the sum of the sizes; the mean's error moves x - mu by
60 u (mean |x|).  r is half that relative plus a few ulps.  So for fp32 output
|dy| <= 1e-5 (|y - b| + |w| r mean|x|) + 2 u |b| is ample; bf16 adds 2^-8 |y|.
dx: r (q - c0 - xh c1) with c0, c1 means of a row: 1e-5 r (|q| + mean|q| +
|xh| mean|q xh|) plus, from xh's own error, its share; bf16 adds 2^-8 |dx|.
Column sums: fp32 sums over N rows in a fixed tree; at most 1,100 in sequence:
|d| <= 1100 u sum|terms| (7e-5), taken as 1e-4 of the sum of sizes.
"""
import math

import pytest
import torch

from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(n, d, dtype, seed, pad=0, start=0, scale=1.0, shift=0.25):
    """[n, d] at a stride of d + pad, `start` elements into an allocation of NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((start + n * (d + pad) + 8,), math.nan, dtype=DT[dtype], device="cuda")
    x = buf[start:start + n * (d + pad)].view(n, d + pad)[:, :d]
    x.copy_(torch.randn((n, d), generator=g, device="cuda") * scale + shift)
    return x


def vectors(d, ptype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    w = 1.0 + 0.3 * torch.randn(d, generator=g, device="cuda")
    b = 0.5 * torch.randn(d, generator=g, device="cuda")
    return w.to(DT[ptype]), b.to(DT[ptype])


def statistics(x, rms, eps):
    x = x.double()
    mu = torch.zeros_like(x[:, :1]) if rms else x.mean(1, keepdim=True)
    return mu, ((x - mu) ** 2).mean(1, keepdim=True).add(eps).rsqrt()


def assert_close(got, ref, bound, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), (what, bad.nonzero()[:5].tolist(), got[bad][:5].tolist(),
                                 ref[bad][:5].tolist(), bound.expand_as(ref)[bad][:5].tolist())


def check_fwd(x, w, b, rms, eps=1e-6, y="new"):
    mu, r = statistics(x, rms, eps)
    wd = torch.ones(x.shape[1], device="cuda").double() if w is None else w.double()
    bd = torch.zeros(x.shape[1], device="cuda").double() if b is None else b.double()
    ref = (x.double() - mu) * r * wd + bd
    size = (ref - bd).abs() + wd.abs() * r * x.double().abs().mean(1, keepdim=True)
    y, stats = T.norm_fwd(x, w, b, rms=rms, eps=eps, y=y)
    bound = 1e-5 * size + 2.0 ** -23 * bd.abs() + 1e-30
    if x.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs()
    assert_close(y, ref, bound, "y")
    assert_close(stats[:, :1], mu, 1e-5 * x.double().abs().mean(1, keepdim=True) + 1e-30, "mu")
    return y, stats


def check_bwd(gy, x, w, rms, eps=1e-6, bias=True, **kw):
    mu, r = statistics(x, rms, eps)
    stats = torch.cat([mu, r], 1).float().contiguous()
    mu, r = stats[:, :1].double(), stats[:, 1:].double()  # as given
    wd = torch.ones(x.shape[1], device="cuda").double() if w is None else w.double()
    g = gy.double().clone()
    xh = (x.double() - mu) * r
    q = g * wd
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    ref = r * ((q if rms else q - mean(q)) - xh * mean(q * xh))
    size = r * (q.abs() + mean(q.abs()) + xh.abs() * mean((q * xh).abs()))
    gx, gw, gb = T.norm_bwd(gy, x, w, stats, rms=rms, grad_bias=bias, **kw)
    if gx is not None:
        bound = 1e-5 * size + 1e-30 + (2.0 ** -8 * ref.abs() if x.dtype == torch.bfloat16 else 0)
        assert_close(gx, ref, bound, "dx")
    if gw is not None:
        assert_close(gw, (g * xh).sum(0), 1e-4 * (g * xh).abs().sum(0) + 1e-30, "dw")
    if gb is not None:
        assert_close(gb, g.sum(0), 1e-4 * g.abs().sum(0) + 1e-30, "db")
    return gx, gw, gb


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 31, 64, 127, 128, 250, 512, 513, 1000, 1024, 1537, 2048, 2049, 4096,
          4097, 5000, 8192, 8193, 16383, 16384]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dtype, rms, gpu):
    for n in (1, 5, 37):
        x = rows(n, d, dtype, d + n)
        w, b = vectors(d, dtype, d)
        check_fwd(x, w, b, rms)
        check_bwd(rows(n, d, dtype, d + n + 1, shift=0.0), x, w, rms)


@pytest.mark.parametrize("n", [1, 2, 63, 1000, 2049, 8300, 20000])
def test_batches(n, gpu):
    for d in (64, 640):
        for rms in (False, True):
            x = rows(n, d, "bf16", n)
            w, b = vectors(d, "f32", d)
            check_fwd(x, w, b, rms)
            check_bwd(rows(n, d, "bf16", n + 1), x, w, rms)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,pad,start", [(1000, 1, 0), (1000, 24, 1), (77, 3, 5), (4100, 0, 7), (2, 1, 1),
                                         (8, 8, 1), (9000, 1, 3)])
def test_starts_strides_and_in_place(d, pad, start, dtype, gpu):
    n = 33
    w, b = vectors(d, dtype, d)
    for rms in (False, True):
        x = rows(n, d, dtype, d, pad, start)
        gy = rows(n, d, dtype, d + 1, 2 * pad, start + 1, shift=0.0)
        buf = torch.full((start + n * (d + pad) + 8,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[start:start + n * (d + pad)].view(n, d + pad)[:, :d]

        def untouched():
            rest = buf.clone()
            rest[start:start + n * (d + pad)].view(n, d + pad)[:, :d] = 7.0
            return bool((rest == 7.0).all())

        check_fwd(x, w, b, rms, y=out)
        assert untouched()
        check_bwd(gy, x, w, rms, grad_x=out)
        assert untouched()
        y = T.norm_fwd(x, w, b, rms=rms)[0]
        stats = T.norm_fwd(x, w, b, rms=rms)[1]
        fresh = T.norm_bwd(gy, x, w, stats, rms=rms)[0]
        over_g, over_x = gy.clone(), x.clone()
        T.norm_bwd(over_g, x, w, stats, rms=rms, grad_x="inplace")
        T.norm_bwd(gy, over_x, w, stats, rms=rms, grad_x=over_x)
        strided = rows(n, d, dtype, d + 1, 2 * pad, start + 1, shift=0.0)
        T.norm_bwd(strided, x, w, stats, rms=rms, grad_x="inplace")
        assert torch.equal(over_g, fresh) and torch.equal(over_x, fresh) and torch.equal(strided, fresh)
        T.norm_fwd(x, w, b, rms=rms, y="inplace")
        assert torch.equal(x, y)


@pytest.mark.parametrize("rms", [False, True])
def test_parameters(rms, gpu):
    """Either type of parameters with either type of rows, and none."""
    for dtype in ("bf16", "f32"):
        for ptype in ("bf16", "f32"):
            x = rows(9, 1001, dtype, 3)
            w, b = vectors(1001, ptype, 4)
            gy = rows(9, 1001, dtype, 5)
            for ww, bb in ((w, b), (w, None), (None, b), (None, None)):
                check_fwd(x, ww, bb, rms)
                check_bwd(gy, x, ww, rms, bias=bb is not None)


def test_values(gpu):
    """Rows far from zero, tiny and huge rows, constant rows, large eps."""
    for dtype in ("bf16", "f32"):
        for scale, shift, eps in ((1.0, 1000.0, 1e-6), (1e-12, 0.0, 0.0), (1e12, 0.0, 1e-6),
                                  (1.0, 0.0, 100.0)):
            x = rows(5, 3000, dtype, 1, scale=scale, shift=shift)
            w, b = vectors(3000, dtype, 2)
            for rms in (False, True):
                check_fwd(x, w, b, rms, eps)
                check_bwd(rows(5, 3000, dtype, 2), x, w, rms, eps)
        x = torch.full((3, 100), 2.5, dtype=DT[dtype], device="cuda")
        y, stats = T.norm_fwd(x, None, None, eps=1e-6)
        assert bool((y == 0).all()) and torch.allclose(stats[:, 1], torch.tensor(1000.0, device="cuda"))
        x[1, 7] = math.nan
        x[2, 9] = math.inf
        y = T.norm_fwd(x)[0]
        assert bool((y[0] == 0).all()) and bool(y[1].isnan().all()) and bool(y[2].isnan().all())


def test_some_outputs_accumulation_and_empty_batches(gpu):
    d = 700
    x, gy = rows(50, d, "bf16", 1), rows(50, d, "bf16", 2)
    w, b = vectors(d, "bf16", 3)
    stats = T.norm_fwd(x, w, b)[1]
    gx, gw, gb = T.norm_bwd(gy, x, w, stats, grad_bias=True)
    only = T.norm_bwd(gy, x, w, stats, grad_weight=False)
    assert torch.equal(only[0], gx) and only[1] is None and only[2] is None
    only = T.norm_bwd(gy, x, w, stats, grad_x=None)
    assert only[0] is None and torch.equal(only[1], gw)
    only = T.norm_bwd(gy, x, w, stats, grad_x=None, grad_weight=None, grad_bias=True)
    assert torch.equal(only[2], gb)
    aw, ab = torch.ones(d, device="cuda"), torch.full((d,), 2.0, device="cuda")
    T.norm_bwd(gy, x, w, stats, grad_weight=aw, grad_bias=ab, accumulate=True)
    assert torch.equal(aw, 1.0 + gw) and torch.equal(ab, 2.0 + gb)
    none = x[:0]
    y, st = T.norm_fwd(none, w, b)
    assert y.shape == (0, d) and st.shape == (0, 2)
    T.norm_bwd(none, none, w, st, grad_weight=aw, grad_bias=ab, accumulate=True)
    assert torch.equal(aw, 1.0 + gw)
    _, zw, zb = T.norm_bwd(none, none, w, st, grad_bias=True)
    assert bool((zw == 0).all()) and bool((zb == 0).all())
    y, st = T.norm_fwd(x, w, b, stats=False)
    assert st is None


def test_same_bits_every_time(gpu):
    x, gy = rows(5000, 1024, "bf16", 1), rows(5000, 1024, "bf16", 2)
    w, b = vectors(1024, "bf16", 3)
    stats = T.norm_fwd(x, w, b)[1]
    first = T.norm_bwd(gy, x, w, stats, grad_bias=True)
    for _ in range(5):
        again = T.norm_bwd(gy, x, w, stats, grad_bias=True)
        assert all(torch.equal(a, c) for a, c in zip(first, again))


def test_central_differences(gpu):
    """The gradients against differences of the definition in 64 bits."""
    n, d = 3, 20
    x = rows(n, d, "f32", 1).double()
    w, b = (t.double() for t in vectors(d, "f32", 2))
    gy = rows(n, d, "f32", 3).contiguous()
    for rms in (False, True):
        def value(x, w, b):
            mu, r = statistics(x, rms, 1e-3)
            return (gy.double() * ((x - mu) * r * w + b)).sum()

        def slope(of, t):
            out, step = torch.empty_like(t), 1e-5
            for i in range(t.numel()):
                e = torch.zeros_like(t).view(-1)
                e[i] = step
                e = e.view_as(t)
                out.view(-1)[i] = (of(t + e) - of(t - e)) / (2 * step)
            return out

        xf, wf, bf = x.float().contiguous(), w.float(), b.float()
        stats = T.norm_fwd(xf, wf, bf, rms=rms, eps=1e-3)[1]
        gx, gw, gb = T.norm_bwd(gy, xf, wf, stats, rms=rms, grad_bias=True)
        for got, ref in ((gx, slope(lambda t: value(t, w, b), x)), (gw, slope(lambda t: value(x, t, b), w)),
                         (gb, slope(lambda t: value(x, w, t), b))):
            # differences: 1e-16 / 1e-5 of values near 60, curvature 1e-10; fp32 sums
            assert bool(((got.double() - ref).abs() <= 2e-5 * (1 + ref.abs())).all())


def test_offsets_past_32_bits(gpu):
    n, d = 140000, 16384
    x = torch.ones((n, d), dtype=torch.bfloat16, device="cuda")
    x[-2:] = rows(2, d, "bf16", 1)
    w, b = vectors(d, "bf16", 2)
    y, stats = T.norm_fwd(x, w, b)
    small, st = T.norm_fwd(x[-2:].clone(), w, b)
    assert torch.equal(y[-2:], small) and torch.equal(stats[-2:], st)
    gx = T.norm_bwd(y, x, w, stats, grad_x="inplace")[0]
    assert torch.equal(gx[-2:], T.norm_bwd(small, x[-2:].clone(), w, st)[0])


def test_graph_replays_equal_eager(gpu):
    n, d = 300, 2048
    x, gy = rows(n, d, "bf16", 1), rows(n, d, "bf16", 2)
    w, b = vectors(d, "bf16", 3)
    y, gx = torch.empty_like(x), torch.empty_like(x)
    stats = torch.empty((n, 2), device="cuda")
    gw, gb = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    ws = T.NormWorkspace(n, d)

    def step():
        T.norm_fwd(x, w, b, y=y, stats=stats)
        T.norm_bwd(gy, x, w, stats, grad_x=gx, grad_weight=gw, grad_bias=gb, workspace=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    for r in range(4):
        x.copy_(rows(n, d, "bf16", 30 + r))
        outs = (y, gx, gw, gb, stats)
        for t in outs:
            t.fill_(3)
        ws.tensor.fill_(r)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        step()
        assert all(torch.equal(a, c) for a, c in zip(got, outs))


def test_binding_refuses(gpu):
    x = rows(4, 100, "bf16", 1)
    w, b = vectors(100, "bf16", 1)
    stats = T.norm_fwd(x, w, b)[1]
    for bad in (lambda: T.norm_fwd(x, w[:99], b), lambda: T.norm_fwd(x, w, b, y=torch.empty_like(x[:3])),
                lambda: T.norm_fwd(x, w, b, y="over"), lambda: T.norm_fwd(x, w.cpu(), b),
                lambda: T.norm_fwd(x, w, b, stats=torch.empty(4, 1, device="cuda")),
                lambda: T.norm_fwd(x.t(), None, None), lambda: T.norm_bwd(x[:3], x, w, stats),
                lambda: T.norm_bwd(x, x, w, stats, accumulate=True),
                lambda: T.norm_bwd(x, x, w, stats[:3].contiguous())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: T.norm_fwd(x.half(), w, b), lambda: T.norm_fwd(x, w, b.float()),
                lambda: T.norm_bwd(x, x, w, stats.double())):
        with pytest.raises(TypeError):
            bad()
    wide = rows(2, 16385, "bf16", 1)
    for bad in (lambda: T.norm_fwd(wide), lambda: T.norm_bwd(wide, wide, None, stats),
                lambda: T.norm_fwd(x, w, b, eps=-1.0), lambda: T.norm_fwd(x, w, b, eps=math.nan),
                lambda: T.norm_bwd(x, x, w, stats, grad_x=None, grad_weight=None)):
        with pytest.raises(T.TurnKLError):
            bad()
