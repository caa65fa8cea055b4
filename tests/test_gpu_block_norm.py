"""turnkl_block_norm_fwd and turnkl_block_norm_bwd against their formulas in 64 bits and
against central differences.

Tolerances (u = 2^-24).  A row's sum takes at most 40 terms in sequence a thread and a tree
of 12 steps, so 60 u of the sum of the sizes: a mean is off by 60 u mean|x|, a
1 / deviation by half the relative error of a mean of squares and three units, 40 u.
Forward: a is off by 50 u (|a| + |w_post| r_f mean|f|), h' by that times |gate| and two
units of its terms; y by what that and its own norm give: with e the error of h',
|dy| <= |w| r (e + mean e) + 50 u (|y - b| + |w| r mean|h'|) + 2 u |b|, and |y - b| times
the relative error of r from e, r sqrt(mean e^2).  For the bound all this is computed in
64 bits with 60 u in place of each number above.  Backward the inputs are given, so each
output is off by 100 u of the sizes of its terms, sums over N rows by at most
(N / 256 + 80) u of the sum of their sizes, at most 500 u here.  bf16 outputs add 2^-8.
"""
import math

import pytest
import torch

from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
TYPES = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")]  # branch, residual


def rows(n, d, dtype, seed, pad=0, start=0, scale=1.0, shift=0.25):
    """[n, d] at a stride of d + pad, `start` elements into an allocation of NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((start + n * (d + pad) + 8,), math.nan, dtype=DT[dtype], device="cuda")
    x = buf[start:start + n * (d + pad)].view(n, d + pad)[:, :d]
    x.copy_(torch.randn((n, d), generator=g, device="cuda") * scale + shift)
    return x


def vector(d, ptype, seed, mean=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    return (mean + 0.3 * torch.randn(d, generator=g, device="cuda")).to(DT[ptype])


def f64(t):
    return None if t is None else t.double()


def mean(t):
    return t.mean(1, keepdim=True)


def moments(x, rms, eps):
    mu = torch.zeros_like(x[:, :1]) if rms else mean(x)
    return mu, (mean((x - mu) ** 2) + eps).rsqrt()


def close(got, ref, bound, what):
    bound = bound.expand_as(ref) + 1e-30
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs()
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(),
                                 ref[bad][:4].tolist(), bound[bad][:4].tolist())


class Case:
    def __init__(self, n, d, types, seed, gate="none", post=False, rms=True, ptype="f32", scale=0.7, pad=0,
                 start=0, eps=1e-6, bias=True):
        ft, rt = types
        self.n, self.d, self.post, self.rms, self.scale, self.eps = n, d, post, rms, scale, eps
        self.gate_kind = gate
        make = lambda t, s, **kw: rows(n, d, t, seed + s, pad, start, **kw)  # noqa: E731
        self.h, self.f = make(rt, 1), make(ft, 2, scale=0.8)
        self.gate = None if gate == "none" else vector(d, ptype, seed + 3, 0.5) if gate == "vector" else \
            make(ft, 3, scale=0.3, shift=0.5)
        self.w, self.b = vector(d, ptype, seed + 4), vector(d, ptype, seed + 5, 0.0) if bias else None
        self.wp = vector(d, ptype, seed + 6) if post else None
        self.gy, self.gh = make(ft, 7, shift=0.0), make(rt, 8, shift=0.1)

    def kw(self):
        return dict(gate=self.gate, post_norm=self.post, post_weight=self.wp, residual_scale=self.scale,
                    rms=self.rms)

    def check_fwd(self, out=None):
        o = 60 * U
        s = float(torch.tensor(self.scale, dtype=torch.float32))
        h, f = self.h.double().clone(), self.f.double().clone()
        gate = 1.0 if self.gate is None else self.gate.double().clone()
        a, ea = f, torch.zeros_like(f)
        if self.post:
            mu, r = moments(f, self.rms, self.eps)
            a = (f - mu) * r * self.wp.double()
            ea = o * (a.abs() + self.wp.double().abs() * r * mean(f.abs()))
            post = torch.cat([mu, r], 1)
            post_err = torch.cat([o * mean(f.abs()), o * r], 1)
        hn = s * h + gate * a
        size = (s * h).abs() + (gate * a).abs()
        e = ea * (gate.abs() if self.gate is not None else 1.0) + 3 * U * size
        mu, r = moments(hn, self.rms, self.eps)
        w = 1.0 if self.w is None else self.w.double()
        b = 0.0 if self.b is None else self.b.double()
        y = (hn - mu) * r * w
        aw = w.abs() if self.w is not None else 1.0
        er = r * r * mean(e * e).sqrt() + o * r
        ey = aw * r * (e + mean(e)) + o * aw * r * mean(hn.abs()) + y.abs() * (er / r) + o * y.abs()
        got = T.block_norm_fwd(self.h, self.f, self.w, self.b, eps=self.eps, out=out, **self.kw())
        close(got.residual, hn, e, "h'")
        close(got.y, y + b, ey + 2 * U * (y + b).abs(), "y")
        close(got.stats, torch.cat([mu, r], 1), torch.cat([mean(e) + o * mean(hn.abs()), er], 1), "stats")
        if self.post:
            close(got.post_stats, post, post_err, "post stats")
        return got

    def given(self):
        """The forward call's outputs, as the gradient takes them (h' is rounded)."""
        hn = self.h
        mu, r = moments(hn.double(), self.rms, self.eps)
        muf, rf = moments(self.f.double(), self.rms, self.eps)
        return hn, torch.cat([mu, r], 1).float(), torch.cat([muf, rf], 1).float() if self.post else None

    def check_bwd(self, use_gh=True, out="new", accumulate=False, **kw):
        hn, stats, post_stats = self.given()
        d = self.d
        s = float(torch.tensor(self.scale, dtype=torch.float32))
        gy, f = self.gy.double().clone(), self.f.double().clone()
        gh = self.gh.double().clone() if use_gh else torch.zeros_like(gy)
        mu, r = stats[:, :1].double(), stats[:, 1:].double()
        w = 1.0 if self.w is None else self.w.double()
        xh = (hn.double() - mu) * r
        # xh's own size of terms: a difference that cancels errs by the larger of its sides
        sx = (hn.double().abs() + mu.abs()) * r
        q = gy * w
        t = gh + r * ((q if self.rms else q - mean(q)) - xh * mean(q * xh))
        st = gh.abs() + r * (q.abs() + mean(q.abs()) + sx * mean((q * sx).abs()))
        gate = torch.ones_like(gy) if self.gate is None else self.gate.double().expand_as(gy).clone()
        ref = {"residual": (s * t, abs(s) * st), "weight": ((gy * xh).sum(0), (gy * sx).abs().sum(0)),
               "bias": (gy.sum(0), gy.abs().sum(0))}
        da, sda = gate * t, gate.abs() * st
        if self.post:
            muf, rf = post_stats[:, :1].double(), post_stats[:, 1:].double()
            wp = self.wp.double()
            fh, sf = (f - muf) * rf, (f.abs() + muf.abs()) * rf
            a, sa = fh * wp, sf * wp.abs()
            p, sp = da * wp, sda * wp.abs()
            df = rf * ((p if self.rms else p - mean(p)) - fh * mean(p * fh))
            ref["branch"] = (df, rf * (sp + mean(sp) + sf * mean(sp * sf)))
            ref["post_weight"] = ((da * fh).sum(0), (sda * sf).sum(0))
        else:
            a, sa = f, f.abs()
            ref["branch"] = (da, sda)
        if self.gate_kind == "matrix":
            ref["gate"] = (t * a, st * sa)
        elif self.gate_kind == "vector":
            ref["gate"] = ((t * a).sum(0), (st * sa).sum(0))
        if out == "new":
            out = T.new_block_norm_grads(self.n, d, self.f.dtype, self.h.dtype, gate=self.gate_kind, bias=True,
                                         post_weight=self.post)
            for x in out:
                if x is not None:
                    x.fill_(math.nan)
        old = [None if x is None else x.double().clone() for x in out]
        got = T.block_norm_bwd(self.gy, self.gh if use_gh else None, hn, stats, self.f, self.w,
                               post_stats=post_stats, out=out, accumulate=accumulate, **self.kw(), **kw)
        for name, x, before in zip(got._fields, got, old):
            if x is None:
                continue
            v, size = ref[name]
            if x.dim() == 1 and accumulate:
                v, size = v + before, size + before.abs()
            close(x, v, (500 if x.dim() == 1 else 100) * U * size, name)
        return got


WIDTHS = [1, 2, 3, 5, 8, 9, 31, 32, 33, 63, 64, 100, 255, 256, 257, 512, 520, 1000, 1537, 2048, 2049, 4096, 4097,
          5120, 8192, 8193, 12000, 16383, 16384]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, types, gpu):
    for n in (1, 5, 37):
        for i, (gate, post, rms) in enumerate((("none", False, True), ("vector", True, False),
                                               ("matrix", True, True), ("matrix", False, False),
                                               ("vector", False, True))):
            c = Case(n, d, types, d + n + i, gate, post, rms, ptype=("f32", "bf16")[i % 2])
            c.check_fwd()
            c.check_bwd()


@pytest.mark.parametrize("n", [2, 3, 63, 1000, 2049, 8300, 20000])
def test_batches(n, gpu):
    for d in (64, 640):
        for types in TYPES[:2]:
            c = Case(n, d, types, n, "vector", True, n % 2 == 0)
            c.check_fwd()
            c.check_bwd()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("pad,start", [(1, 0), (5, 3), (0, 1), (8, 8)])
def test_strides_and_starts(pad, start, types, gpu):
    for d in (5, 64, 777, 4100, 8200):
        c = Case(19, d, types, d, "matrix", True, False, pad=pad, start=start)
        out = T.BlockNorm(rows(19, d, types[1], 1, pad, start), rows(19, d, types[0], 1, pad, start),
                          torch.empty((19, 2), device="cuda"), torch.empty((19, 2), device="cuda"))
        c.check_fwd(out)
        grads = T.BlockNormGrads(rows(19, d, types[1], 1, pad, start), rows(19, d, types[0], 1, pad, start),
                                 rows(19, d, types[0], 1, pad, start),
                                 *[torch.empty(d, device="cuda") for _ in range(3)])
        c.check_bwd(out=grads)
        for x in (out.residual, out.y, *grads[:3]):  # nothing outside the rows is written
            whole = torch.empty(0, dtype=x.dtype, device="cuda").set_(x.untyped_storage())
            left = torch.ones(whole.numel(), dtype=torch.bool, device="cuda")
            for i in range(19):
                left[start + i * (d + pad):start + i * (d + pad) + d] = False
            assert bool(whole[left].isnan().all())


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("d", [33, 300, 4097, 9000])
def test_in_place(d, types, gpu):
    for post in (False, True):
        kw = dict(gate="vector", post=post, rms=False)
        want = Case(23, d, types, 1, **kw).check_fwd()
        c = Case(23, d, types, 1, **kw)
        got = T.block_norm_fwd(c.h, c.f, c.w, c.b, out=T.BlockNorm(c.h, c.f, None, None), **c.kw())
        assert got.residual is c.h and torch.equal(got.residual, want.residual) and torch.equal(got.y, want.y)
        c = Case(23, d, types, 1, **kw)
        want = c.check_bwd()
        hn, stats, post_stats = c.given()
        out = T.BlockNormGrads(c.gh, c.gy, *want[2:])
        got = T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, c.w, post_stats=post_stats,
                               out=T.BlockNormGrads(*out[:2], *[None if x is None else x.clone() for x in out[2:]]),
                               **c.kw())
        for a, b in zip(got, want):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("d", [40, 600, 3001, 9000])
def test_without_parameters_and_parts(d, gpu):
    for types in TYPES:
        c = Case(11, d, types, d, bias=False)
        c.w = None
        c.check_fwd()
        c.check_bwd(use_gh=False)
        c = Case(11, d, types, d, "vector", True, False)
        full = c.check_bwd()
        for i in range(6):  # each alone
            out = T.BlockNormGrads(*[torch.full_like(x, 7.0) if j == i else None for j, x in enumerate(full)])
            got = c.check_bwd(out=out)
            assert torch.equal(got[i], full[i])


@pytest.mark.parametrize("d", [64, 700, 4096, 10000])
def test_accumulate(d, gpu):
    c = Case(50, d, ("bf16", "bf16"), d, "vector", True, False)
    out = T.new_block_norm_grads(50, d, gate="vector", bias=True, post_weight=True)
    for x in out:
        x.fill_(3.0)
    c.check_bwd(out=out, accumulate=True)


def test_no_rows(gpu):
    c = Case(0, 40, ("bf16", "f32"), 1, "matrix", True)
    c.check_fwd()
    got = c.check_bwd()
    assert not bool(got.weight.any()) and not bool(got.bias.any()) and not bool(got.post_weight.any())
    out = T.BlockNormGrads(*got[:3], *[torch.full((40,), 2.0, device="cuda") for _ in range(3)])
    c.check_bwd(out=out, accumulate=True)
    assert bool((out.weight == 2).all())


@pytest.mark.parametrize("d", [48, 520, 9000])
def test_rows_without_variance_and_values_that_are_no_numbers(d, gpu):
    h, f = torch.full((4, d), 3.0, device="cuda"), torch.full((4, d), -2.0, device="cuda")
    got = T.block_norm_fwd(h, f, gate=torch.ones(d, device="cuda"), post_norm=True)
    assert not bool(got.y.any()) and bool((got.residual == 3.0).all())
    assert bool((got.stats[:, 1] - 1e3).abs().max() < 1e-3)
    h[1, 5], f[2, 7] = math.inf, math.nan
    got = T.block_norm_fwd(h, f)
    assert bool(got.residual[1, 5] == math.inf) and bool(got.y[1].isnan().any()) and bool(got.y[2].isnan().all())
    assert bool(got.y[0].isfinite().all()) and bool(got.y[3].isfinite().all())
    w = torch.ones(d, device="cuda")
    g = torch.ones((4, d), device="cuda")
    stats = torch.tensor([[0.0, 1.0]] * 4, device="cuda")
    g[1, 3] = math.inf
    out = T.block_norm_bwd(g, None, torch.ones((4, d), device="cuda"), stats, f, w)
    assert bool(out.residual[1].isnan().any()) and bool(out.residual[0].isfinite().all())
    assert bool(out.weight[3] == math.inf) and bool(out.weight[:3].isfinite().all())


def test_the_same_bits_from_call_to_call(gpu):
    for d in (100, 1024, 4096, 9000):
        c = Case(3000, d, ("bf16", "bf16"), 5, "vector", True, False)
        first = c.check_bwd()
        ws = T.BlockNormWorkspace(5000, d)
        for _ in range(3):
            ws.tensor.random_(0, 255)
            for a, b in zip(c.check_bwd(workspace=ws), first):
                assert torch.equal(a, b)


def test_differences(gpu):
    """The gradient of L = sum(cy y) + sum(ch h') against central differences of the 64-bit
    formula at the kernel's inputs: step 1e-5 of numbers of size one leaves 1e-9."""
    torch.manual_seed(1)
    n, d, eps = 3, 12, 1e-6
    for gate in ("none", "vector", "matrix"):
        for post in (False, True):
            for rms in (False, True):
                c = Case(n, d, ("f32", "f32"), 9, gate, post, rms, eps=eps)
                fwd = T.block_norm_fwd(c.h, c.f, c.w, c.b, eps=eps, **c.kw())
                out = T.new_block_norm_grads(n, d, torch.float32, gate=gate, bias=True, post_weight=post)
                T.block_norm_bwd(c.gy, c.gh, fwd.residual, fwd.stats, c.f, c.w, post_stats=fwd.post_stats,
                                 out=out, **c.kw())
                s = float(torch.tensor(c.scale, dtype=torch.float32))
                names = {"residual": c.h, "branch": c.f, "gate": c.gate, "weight": c.w, "bias": c.b,
                         "post_weight": c.wp}
                base = {k: f64(v) for k, v in names.items()}

                def loss(v):
                    a = v["branch"]
                    if post:
                        mu, r = moments(a, rms, eps)
                        a = (a - mu) * r * v["post_weight"]
                    h = s * v["residual"] + (a if v["gate"] is None else a * v["gate"])
                    mu, r = moments(h, rms, eps)
                    return float((c.gy.double() * ((h - mu) * r * v["weight"] + v["bias"])).sum()
                                 + (c.gh.double() * h).sum())

                for name in names:
                    got = getattr(out, name)
                    if got is None:
                        continue
                    for at in ([(0, 0), (2, 7), (1, 11)] if base[name].dim() == 2 else [(0,), (5,), (11,)]):
                        moved = []
                        for sign in (1, -1):
                            v = dict(base)
                            v[name] = base[name].clone()
                            v[name][at] += sign * 1e-5
                            moved.append(loss(v))
                        want = (moved[0] - moved[1]) / 2e-5
                        assert abs(float(got[at]) - want) < 2e-4, (gate, post, rms, name, at, float(got[at]), want)


def test_graph_replays(gpu):
    for d in (200, 2048, 9000):
        c = Case(100, d, ("bf16", "f32"), 3, "matrix", True, False)
        fwd = c.check_fwd()
        out = T.new_block_norm_grads(100, d, torch.bfloat16, torch.float32, gate="matrix", bias=True, post_weight=True)
        ws = T.BlockNormWorkspace(100, d)

        def call():
            o = T.block_norm_fwd(c.h, c.f, c.w, c.b, out=fwd, **c.kw())
            T.block_norm_bwd(c.gy, c.gh, o.residual, o.stats, c.f, c.w, post_stats=o.post_stats, out=out,
                             workspace=ws, **c.kw())

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for r in range(4):
            c.f.copy_(rows(100, d, "bf16", 50 + r))
            graph.replay()
            got = [x.clone() for x in (*fwd, *out)]
            for x in (*fwd, *out):
                x.fill_(math.nan)
            torch.cuda.synchronize()
            call()
            for a, b in zip(got, (*fwd, *out)):
                assert torch.equal(a, b)


def test_streams(gpu):
    made = []
    for i in range(2):
        c = Case(4000, 1024, ("bf16", "bf16"), i, "vector", True, True)
        hn, stats, post_stats = c.given()
        want = c.check_bwd()
        made.append((c, hn, stats, post_stats, want, T.new_block_norm_grads(4000, 1024, gate="vector", bias=True,
                                                                           post_weight=True),
                     T.BlockNormWorkspace(4000, 1024), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for c, hn, stats, post_stats, _, out, ws, stream in made:
            with torch.cuda.stream(stream):
                T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, c.w, post_stats=post_stats, out=out, workspace=ws,
                                 **c.kw())
    torch.cuda.synchronize()
    for *_, want, out, _, _ in made:
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_offsets_past_32_bits(gpu):
    n, d = 280000, 8192  # 4.6 GB a matrix
    h = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    f = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    f[-1, ::2] = 2.0
    out = T.block_norm_fwd(h, f, rms=True, out=T.BlockNorm(h, f, torch.empty((n, 2), device="cuda"), None))
    assert bool((out.residual[-1, ::2] == 2).all()) and not bool(out.residual[-1, 1::2].any())
    assert bool((out.y[-1, ::2].float() - 2 ** 0.5).abs().max() < 0.01)
    assert not bool(out.y[:5].any()) and not bool(out.y[n - 6:n - 1].any())
    del out
    g = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    g[-1] = 1.0
    stats = torch.zeros((n, 2), device="cuda")
    stats[:, 1] = 1.0
    h.zero_()
    got = T.block_norm_bwd(g, None, h, stats, f, None, rms=True,
                           out=T.BlockNormGrads(None, g, None, None, torch.empty(d, device="cuda"), None))
    assert bool((got.branch[-1] == 1).all()) and not bool(got.branch[n - 4:n - 1].any())
    assert bool((got.bias == 1).all())


def test_refusals(gpu):
    c = Case(6, 32, ("bf16", "f32"), 1, "vector", True)
    hn, stats, post_stats = c.given()
    d64 = torch.zeros((6, 32), dtype=torch.float64, device="cuda")
    for call in (lambda: T.block_norm_fwd(c.h[:5], c.f), lambda: T.block_norm_fwd(c.h, c.f, c.w[:5]),
                 lambda: T.block_norm_fwd(c.h, c.f, gate=c.h), lambda: T.block_norm_fwd(c.h, c.f.cpu()),
                 lambda: T.block_norm_fwd(c.h, c.f, out=T.BlockNorm(c.f, c.f, None, None)),
                 lambda: T.block_norm_bwd(c.gy[:5], None, hn, stats, c.f, None),
                 lambda: T.block_norm_bwd(c.gy, c.gh, hn, stats[:5], c.f, None),
                 lambda: T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, None, accumulate=True)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: T.block_norm_fwd(d64, c.f),
                 lambda: T.block_norm_fwd(c.h, c.f, c.w, c.b.bfloat16())):
        with pytest.raises(TypeError):
            call()
    for code, call in (
            (T.ERR_INVALID_ARG, lambda: T.block_norm_fwd(c.f, c.h)),  # fp32 branches on a bf16 stream
            (T.ERR_INVALID_ARG, lambda: T.block_norm_fwd(c.h, c.f, post_weight=c.wp)),
            (T.ERR_INVALID_ARG, lambda: T.block_norm_fwd(c.h, c.f, residual_scale=math.nan)),
            (T.ERR_INVALID_ARG, lambda: T.block_norm_fwd(c.h, c.f, eps=-1.0)),
            (T.ERR_INVALID_ARG, lambda: T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, None, post_norm=True)),
            (T.ERR_ALIAS, lambda: T.block_norm_fwd(
                c.h, c.f, out=T.BlockNorm(c.h, c.f, c.h.view(-1)[:12].view(6, 2), None))),
            (T.ERR_ALIAS, lambda: T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, None, out=T.BlockNormGrads(
                hn, None, None, None, None, None))),
            (T.ERR_WORKSPACE, lambda: T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, None,
                                                       workspace=T.BlockNormWorkspace(1, 4)))):
        with pytest.raises(T.TurnKLError) as e:
            call()
        assert e.value.code == code, (e.value.code, code)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("d,post", [(40, True), (700, False), (4097, True), (8192, False), (8193, False), (16384, True)])
def test_no_rows_of_every_form(d, post, types, gpu):
    """The sums over no rows are zeros, or what was there, whatever the workspace holds."""
    c = Case(0, d, types, 1, "vector", post)
    hn, stats, post_stats = c.given()
    ws = T.BlockNormWorkspace(300, d)
    for accumulate in (False, True):
        ws.tensor.fill_(0xFF)  # NaN
        out = T.new_block_norm_grads(0, d, c.f.dtype, c.h.dtype, gate="vector", bias=True, post_weight=post)
        sums = [x for x in out if x is not None and x.dim() == 1]
        assert len(sums) == (4 if post else 3)
        for x in sums:
            x.copy_(torch.arange(d))
        T.block_norm_bwd(c.gy, c.gh, hn, stats, c.f, c.w, post_stats=post_stats, out=out, accumulate=accumulate,
                         workspace=ws, **c.kw())
        for x in sums:
            assert torch.equal(x, torch.arange(d, device="cuda") * (1.0 if accumulate else 0.0))
