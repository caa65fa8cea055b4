"""turnkl_sample_tokens against its definition in 64 bits: sorted logits, running sums.

Tokens are compared exactly: the random numbers are not chosen near a border, and the
chance that one of them lies within 1e-12 of one by itself is below 1e-6 for all tests
together.  logq and logp: the kernel's sums of exp(z - M) are float within a segment of
2,048 (32 terms in sequence a lane, a tree of 6, an exponential's 2 units and its argument's
half: 45 units of 2^-24), all else is double, and both outputs are rounded to float once:
|d| <= 3e-6 + 2^-23 |log|.
"""
import decimal
import math
from decimal import Decimal
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def logits(n, v, dtype, seed, spread=3.0, peak=8.0, pad=0, start=0):
    """[n, v] at a stride of v + pad, `start` elements into an allocation of NaN."""
    buf = torch.full((start + n * (v + pad) + 8,), math.nan, dtype=DT[dtype], device="cuda")
    z = buf[start:start + n * (v + pad)].view(n, v + pad)[:, :v]
    a = torch.randn((n, v), generator=gen(seed), device="cuda") * spread
    at = torch.randint(0, v, (n, min(v, 6)), generator=gen(seed + 1), device="cuda")
    a.scatter_add_(1, at, torch.full_like(at, 1, dtype=torch.float32) * peak)
    z.copy_(a)
    return z


def uniforms(n, seed):
    return torch.rand(n, generator=gen(seed + 7), device="cuda", dtype=torch.float64)


def column(x, n):
    t = torch.as_tensor(x, device="cuda")
    return t.to(torch.float32).double().expand(n)[:, None]


def reference(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens, logq, logp) of rows that hold a finite logit and no NaN."""
    n, v = z.shape
    a = z.double()
    value, col = a.sort(dim=1, descending=True, stable=True)
    heat, k, p, mp = (column(x, n) for x in (temperature, top_k, top_p, min_p))
    greedy = (heat == 0) | (p == 0)
    heat = torch.where(heat == 0, 1.0, heat)
    k = torch.where(greedy, 1, k)
    p = torch.where(greedy, 1.0, p)
    mp = torch.where(greedy, 0.0, mp.clamp(max=1.0))
    w = ((value - value[:, :1]) / heat).exp()
    rank = torch.arange(v, device="cuda").expand(n, v)
    keep = (rank < k) | (k <= 0)
    mass = torch.where(keep, w, 0.0)
    before = mass.cumsum(1) - mass
    keep = keep & ((before < p * mass.sum(1, keepdim=True)) | (p >= 1))
    keep = (keep & (w >= mp)) | (rank == 0)
    q = torch.zeros_like(w).scatter_(1, col, torch.where(keep, w, 0.0))
    run = q.cumsum(1)
    total = run[:, -1:]
    last = torch.where(q > 0, rank, -1).amax(1)
    t = torch.minimum((run <= u[:, None] * total).sum(1), last)[:, None]
    m = value[:, :1]
    logq = (q.gather(1, t).log() - total.log())[:, 0]
    logp = (a.gather(1, t) - m)[:, 0] - (a - m).exp().sum(1).log()
    return t[:, 0].int(), logq, logp


def close(got, ref, what):
    err = (got.double() - ref).abs()
    bound = 3e-6 + 2.0 ** -23 * ref.abs()
    assert bool((err <= bound).all()), (what, float((err - bound).max()))


def check(z, u, **kw):
    got = T.sample_tokens(z, u, **kw)
    ids, logq, logp = reference(z, u, **kw)
    bad = (got.ids != ids).nonzero()[:, 0]
    assert bad.numel() == 0, (bad[:5].tolist(), got.ids[bad][:5].tolist(), ids[bad][:5].tolist(), kw)
    close(got.logq, logq, "logq")
    close(got.logp, logp, "logp")
    return got


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=5), dict(top_k=40, top_p=0.9, temperature=0.8), dict(top_p=0.5),
           dict(top_p=0.95), dict(top_p=0.999, temperature=1.5), dict(min_p=0.05), dict(min_p=1e-4, temperature=1.3),
           dict(top_p=0.9, min_p=0.02), dict(top_k=700, top_p=0.97, min_p=0.001, temperature=1.2), dict(temperature=0.0),
           dict(top_k=1)]
SIZES = [1, 2, 3, 7, 8, 9, 63, 64, 65, 511, 1000, 2047, 2048, 2049, 4097, 32000, 50257, 151936, 151937]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", SIZES)
def test_sizes(v, dtype, gpu):
    z = logits(7, v, dtype, v)
    for i, kw in enumerate(FILTERS):
        check(z, uniforms(7, v + i), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_flat_rows(dtype, gpu):
    """Supports of thousands of tokens, beyond what the lists hold."""
    z = logits(6, 60000, dtype, 5, spread=0.5, peak=0.0)
    for i, kw in enumerate((dict(), dict(top_p=0.9), dict(top_p=0.05), dict(top_p=0.004), dict(top_k=3000),
                            dict(top_k=20000), dict(top_k=20000, top_p=0.7), dict(min_p=0.3), dict(min_p=0.01),
                            dict(top_p=0.5, min_p=0.4), dict(top_k=600), dict(top_k=5000, min_p=0.3))):
        check(z, uniforms(6, i), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_logits(dtype, gpu):
    """Ties at every border: the lower ids stay."""
    n, v = 5, 10000
    z = torch.zeros((n, v), dtype=DT[dtype], device="cuda")
    z[:, 4000:9000] = 1.5
    for i, kw in enumerate((dict(), dict(top_k=10), dict(top_k=4999), dict(top_k=5000), dict(top_k=5001), dict(top_p=0.3),
                            dict(top_p=0.97), dict(min_p=0.5), dict(min_p=1.0), dict(min_p=7.0),
                            dict(top_k=9000, top_p=0.5), dict(top_p=0.02), dict(temperature=0.0))):
        check(z, uniforms(n, i), **kw)
    z.zero_()
    for kw in (dict(), dict(top_k=7), dict(top_p=0.5), dict(top_k=600), dict(top_k=1000, top_p=0.25)):
        check(z, uniforms(n, 3), **kw)
    # numbers exactly on a border belong to what follows it
    z = torch.zeros((8, 4), dtype=DT[dtype], device="cuda")
    u = torch.tensor([0.0, 0.2499, 0.25, 0.4999, 0.5, 0.75, 0.999, 1 - 2.0 ** -53], dtype=torch.float64, device="cuda")
    assert T.sample_tokens(z, u).ids.tolist() == [0, 0, 1, 1, 2, 3, 3, 3]
    assert T.sample_tokens(z, u, top_k=2).ids.tolist() == [0, 0, 0, 0, 1, 1, 1, 1]
    assert T.sample_tokens(z, u, top_p=0.5).ids.tolist() == [0, 0, 0, 0, 1, 1, 1, 1]


def test_every_token_of_a_small_row(gpu):
    """The token where a random number lies in the middle of each token's share."""
    z = logits(1, 40, "f32", 3, peak=2.0)
    for kw in (dict(), dict(top_k=6), dict(top_p=0.8), dict(min_p=0.1, temperature=2.0)):
        w = ((z.double() - z.double().max()) / kw.get("temperature", 1.0)).exp()[0]
        order = w.sort(dim=0, descending=True, stable=True)
        n = kw.get("top_k", 40)
        if "top_p" in kw:
            n = int((order.values.cumsum(0) - order.values < float(torch.tensor(0.8)) * w.sum()).sum())
        if "min_p" in kw:
            n = int((w >= 0.1).sum())
        ids = order.indices[:n].sort().values
        q = w[ids] / w[ids].sum()
        u = q.cumsum(0) - q / 2
        got = T.sample_tokens(z.expand(n, 40).contiguous(), u, **kw)
        assert got.ids.tolist() == ids.tolist()
        close(got.logq, q.log(), "logq")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,start", [(1, 0), (5, 3), (0, 1), (56, 0)])
def test_strides_and_starts(pad, start, dtype, gpu):
    for v in (5, 1000, 2048, 10001):
        z = logits(9, v, dtype, v, pad=pad, start=start)
        for i, kw in enumerate(FILTERS):
            check(z, uniforms(9, i), **kw)


@pytest.mark.parametrize("n", [1, 64, 500, 3000])
def test_batches_with_parameters_of_their_own(n, gpu):
    for v in (700, 20000):
        z = logits(n, v, "bf16", n)
        r = torch.rand((4, n), generator=gen(n), device="cuda")
        kw = dict(temperature=torch.where(r[0] < 0.1, 0.0, 2 * r[0]), top_k=(r[1] * 300 - 50).int(),
                  top_p=torch.where(r[2] < 0.3, 1.0, r[2]).contiguous(), min_p=torch.where(r[3] < 0.5, 0.0, r[3] / 9))
        check(z, uniforms(n, 1), **kw)


def test_masks(gpu):
    z = logits(50, 3000, "bf16", 1)
    mask = (torch.rand(50, generator=gen(1), device="cuda") < 0.5).to(torch.uint8)
    u = uniforms(50, 1)
    want = T.sample_tokens(z, u, top_p=0.9)
    z[mask == 0] = math.nan  # not read
    u[mask == 0] = 5.0
    got = T.sample_tokens(z, u, top_p=0.9, mask=mask)
    on = mask != 0
    assert torch.equal(got.ids[on], want.ids[on]) and torch.equal(got.logq[on], want.logq[on])
    assert bool((got.ids[~on] == -1).all()) and not bool(got.logq[~on].any()) and not bool(got.logp[~on].any())
    got = T.sample_tokens(z, u, mask=torch.zeros_like(mask))
    assert bool((got.ids == -1).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forbidden_tokens_and_empty_rows(dtype, gpu):
    for v in (50, 5000, 151936):
        z = logits(8, v, dtype, v)
        z[:, ::3] = -math.inf
        z[3, :] = -math.inf
        z[3, v // 2] = -4.0  # one allowed token
        z[4, 10:] = -math.inf  # fewer than k
        for i, kw in enumerate(FILTERS):
            check(z, uniforms(8, i), **kw)
        low = torch.finfo(DT[dtype]).min
        z = logits(8, v, dtype, v)
        z[:, 1::2] = low
        z[2] = low  # all equal
        for i, kw in enumerate(FILTERS):
            check(z, uniforms(8, i), **kw)
        z = logits(6, v, dtype, v)
        z[1] = -math.inf
        z[2, 7], z[3, 9], z[4, v - 1] = math.inf, math.nan, math.nan
        for kw in FILTERS:
            got = T.sample_tokens(z, uniforms(6, 1), **kw)
            assert got.ids[1:5].tolist() == [-1] * 4 and min(int(got.ids[0]), int(got.ids[5])) >= 0
            assert bool((got.logq[1] == -math.inf) & (got.logp[1] == -math.inf))
            assert bool(got.logq[2:5].isnan().all()) and bool(got.logp[2:5].isnan().all())


def test_large_and_small_numbers(gpu):
    for off in (-1e4, 1e6, 1e30):
        z = logits(4, 5000, "f32", 2) + off
        for kw in (dict(), dict(top_k=9), dict(top_p=0.9), dict(min_p=0.1)):
            check(z, uniforms(4, 2), **kw)
    z = logits(4, 5000, "f32", 2)
    for heat in (1e-30, 1e-3, 1e3, 1e30):
        for kw in (dict(), dict(top_k=9), dict(top_p=0.9), dict(min_p=0.5)):
            check(z, uniforms(4, 2), temperature=heat, **kw)
    z = torch.full((2, 3000), 3e38, device="cuda")
    z[0, 100:] = -3e38
    check(z, uniforms(2, 1))


def test_bad_rows_are_reported(gpu):
    z, u = logits(9, 400, "bf16", 1), uniforms(9, 1)
    good = T.sample_tokens(z, u)
    ws = T.SampleWorkspace(9, 400)
    nan = math.nan
    for kw, at in ((dict(temperature=[1.0, -1.0, 1, 1, 1, 1, 1, nan, math.inf]), (1, 7, 8)),
                   (dict(top_p=[1.0, 1, 1, 1, -0.5, 1, 1, 1, nan]), (4, 8)), (dict(min_p=[nan, 0, 0, 0, 0, 0, 0, 0, -1.0]), (0, 8))):
        kw = {k: torch.tensor(x, device="cuda") for k, x in kw.items()}
        with pytest.raises(T.TurnKLError) as e:
            T.sample_tokens(z, u, workspace=ws, **kw)
        assert e.value.code == T.ERR_SAMPLING
        got = T.sample_tokens(z, u, workspace=ws, check=False, **kw)
        for i in range(9):
            if i in at:
                assert int(got.ids[i]) == -1 and bool(got.logq[i].isnan())
            else:
                assert int(got.ids[i]) == int(good.ids[i])
    for x in (-0.1, 1.0, nan, math.inf):
        w = u.clone()
        w[5] = x
        got = T.sample_tokens(z, w, workspace=ws, check=False)
        assert int(got.ids[5]) == -1 and ws.status() == T.ERR_SAMPLING
    assert torch.equal(T.sample_tokens(z, u, workspace=ws).ids, good.ids)  # the status is the last call's


def test_outputs_that_are_not_asked_for(gpu):
    z, u = logits(30, 3000, "bf16", 1), uniforms(30, 1)
    for kw in FILTERS:
        full = T.sample_tokens(z, u, **kw)
        part = T.sample_tokens(z, u, out=T.SampledTokens(torch.empty_like(full.ids), None, None), **kw)
        assert torch.equal(part.ids, full.ids)


def test_no_rows(gpu):
    got = T.sample_tokens(torch.empty((0, 50), device="cuda"), uniforms(0, 1))
    assert got.ids.numel() == 0


def test_the_same_bits_from_call_to_call(gpu):
    z, u = logits(40, 60000, "bf16", 1, spread=1.0), uniforms(40, 1)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=3000), dict(top_k=50), dict(min_p=0.01)):
        first = T.sample_tokens(z, u, **kw)
        ws = T.SampleWorkspace(100, 70000)
        for _ in range(3):
            ws.tensor.random_(0, 255)
            got = T.sample_tokens(z, u, workspace=ws, **kw)
            assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_graph_replays(gpu):
    n, v = 20, 30000
    z, u = logits(n, v, "bf16", 1), uniforms(n, 1)
    out, ws = T.new_sampled_tokens(n), T.SampleWorkspace(n, v)
    heat = torch.full((n,), 0.9, device="cuda")
    call = lambda: T.sample_tokens(z, u, temperature=heat, top_p=0.9, out=out, workspace=ws, check=False)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for r in range(4):
        z.copy_(logits(n, v, "bf16", 30 + r))
        u.copy_(uniforms(n, 30 + r))
        heat.fill_(0.5 + 0.2 * r)
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        call()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
        assert torch.equal(out.ids, reference(z, u, heat, 0, 0.9)[0])


def test_streams(gpu):
    made = []
    for i in range(2):
        z, u = logits(64, 50000, "bf16", i), uniforms(64, i)
        made.append((z, u, T.sample_tokens(z, u, top_p=0.9), T.new_sampled_tokens(64), T.SampleWorkspace(64, 50000),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for z, u, _, out, ws, stream in made:
            with torch.cuda.stream(stream):
                T.sample_tokens(z, u, top_p=0.9, out=out, workspace=ws, check=False)
    torch.cuda.synchronize()
    for _, _, want, out, _, _ in made:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_offsets_past_32_bits(gpu):
    n, v = 16000, 151936  # 4.9 GB
    z = torch.full((n, v), -3.0, dtype=torch.bfloat16, device="cuda")
    z[-1, 151000], z[0, 5] = 20.0, 20.0
    u = torch.full((n,), 0.5, dtype=torch.float64, device="cuda")
    for kw in (dict(), dict(top_k=20)):
        got = T.sample_tokens(z, u, **kw)
        assert int(got.ids[-1]) == 151000 and int(got.ids[0]) == 5
        assert int(got.ids[7000]) == (75968 if not kw else 10)


def test_the_largest_vocabulary(gpu):
    v = 2 ** 24
    z = torch.randn((2, v), generator=gen(1), device="cuda").bfloat16()
    for kw in (dict(), dict(top_k=100), dict(top_p=0.001), dict(min_p=0.5)):
        check(z, uniforms(2, 1), **kw)


def test_agrees_with_token_logprobs(gpu):
    z, u = logits(200, 32000, "bf16", 1), uniforms(200, 1)
    got = T.sample_tokens(z, u, top_k=50)
    again = T.token_logprobs(z, got.ids, k=50)
    assert float((again.logp - got.logp).abs().max()) < 1e-5
    assert bool((again.top_ids == got.ids[:, None]).any(1).all())


def test_refusals(gpu):
    z, u = logits(4, 50, "bf16", 1), uniforms(4, 1)
    for call in (lambda: T.sample_tokens(z, u.float()), lambda: T.sample_tokens(z, u[:3]),
                 lambda: T.sample_tokens(z, u.cpu()), lambda: T.sample_tokens(z, u, top_k=torch.ones(4, device="cuda")),
                 lambda: T.sample_tokens(z, u, top_p=torch.ones(3, device="cuda")), lambda: T.sample_tokens(z.t(), u)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        T.sample_tokens(z.half(), u)
    for kw in (dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(top_p=-0.1),
               dict(top_p=math.nan), dict(min_p=-1.0)):
        with pytest.raises(T.TurnKLError) as e:
            T.sample_tokens(z, u, **kw)
        assert e.value.code == T.ERR_INVALID_ARG
    with pytest.raises(T.TurnKLError) as e:
        T.sample_tokens(logits(40, 50000, "bf16", 1), uniforms(40, 1), workspace=T.SampleWorkspace(4, 50))
    assert e.value.code == T.ERR_WORKSPACE
    whole = torch.zeros(8, device="cuda")
    with pytest.raises(T.TurnKLError) as e:
        T.sample_tokens(z, u, out=T.SampledTokens(torch.empty(4, dtype=torch.int32, device="cuda"), whole[:4], whole[2:6]))
    assert e.value.code == T.ERR_ALIAS


@pytest.mark.parametrize("kw", [dict(top_k=50, temperature=0.7), dict(min_p=0.01), dict(temperature=1.3), dict()])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_log_p_of_a_token_with_nearly_all_of_a_row(dtype, kw, gpu):
    """log p = -log(1 + s) for the others' sum s is accurate relative to itself.  The logits
    are multiples of 1/8, so that their differences are exact: 2^-23 for an exponential,
    2^-24 for its correction and for the output, and what the 64-bit sums add: 2^-21."""
    n, v = 40, 20011
    z = (torch.randn(n, v, device="cuda", generator=gen(5)) * 16).round().clamp(-64, 64) / 8
    z[torch.arange(n), torch.arange(n) * 7] = torch.arange(n, device="cuda") / 8 + 17.0
    z = z.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    u = torch.full((n,), 0.5, dtype=torch.float64, device="cuda")
    got = T.sample_tokens(z, u, **kw)
    ids = torch.arange(n, device="cuda") * 7
    rest = z.double() - z.double().amax(1, keepdim=True)
    rest[torch.arange(n), ids] = -math.inf
    ref = -torch.log1p(rest.exp().sum(1))
    assert bool((got.ids == ids).sum() > n // 2)
    took = got.ids == ids
    assert bool(((got.logp.double() - ref).abs() <= 2.0 ** -21 * ref.abs())[took].all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [50, 2048, 2049, 5000, 151936])
def test_the_highest_temperatures(v, dtype, gpu):
    """Forbidden tokens, and the places behind a row's end, weigh nothing where all others
    weigh the same."""
    n = 6
    z = logits(n, v, dtype, v)
    z[:, ::3] = -math.inf
    z[2, 1:-1], z[2, -1] = -math.inf, 1.0
    z[3] = logits(1, v, dtype, 1)[0]
    z[4, -1] = -3e38
    for heat in (4.7e35, 5e35, 1e36, 3e38, 3.4028234e38):
        for i, kw in enumerate((dict(), dict(top_p=0.9), dict(top_k=9), dict(top_k=900, top_p=0.7), dict(min_p=0.3))):
            check(z, uniforms(n, i), temperature=heat, **kw)
        ends = torch.tensor([0.0, 1 - 2.0 ** -53] * (n // 2), dtype=torch.float64, device="cuda")
        check(z, ends, temperature=heat)
        check(z, ends, temperature=torch.full((n,), heat, device="cuda"), top_p=0.99)


@pytest.mark.parametrize("n,repeats,kw", [
    (3000, 2, dict()), (3000, 4, dict()), (200, 2, dict()), (3000, 2, dict(min_p=1e-5)), (250, 2, dict(min_p=1e-5)),
    (3000, 4, dict(min_p=1e-5, temperature=1.7)), (40, 256, dict()), (40, 256, dict(min_p=1e-5))])
def test_random_numbers_on_a_border_between_segments(n, repeats, kw, gpu):
    """Rows of the same segments over and over, some of them without a token, and random
    numbers that lie exactly between two repetitions: the first token behind the border
    follows from the definition, the last one before it from a rounding; nothing else does.
    256 repetitions are more segments than the workgroup that picks has threads."""
    period, filled = 5, 3
    v = repeats * period * 2048
    z = torch.full((n, repeats, period * 2048), -math.inf, device="cuda")
    each = 300 if repeats < 9 else 4
    at = torch.rand((n, filled, 2048), generator=gen(repeats), device="cuda").topk(each, dim=2).indices
    at += torch.arange(filled, device="cuda")[:, None] * 2048
    at = at.reshape(n, 1, -1).expand(n, repeats, -1)
    z.scatter_(2, at, (-2 * torch.rand((n, 1, filled * each), generator=gen(n), device="cuda")).expand(at.shape).contiguous())
    first, last = at[:, 0].amin(1), at[:, 0].amax(1)
    z = z.view(n, v)
    for k in {1, repeats // 2, repeats - 1}:
        u = torch.full((n,), k / repeats, dtype=torch.float64, device="cuda")
        got = T.sample_tokens(z, u, **kw)
        behind, before = first + k * period * 2048, last + (k - 1) * period * 2048
        good = (got.ids == behind) | (got.ids == before)
        assert bool(good.all()), (k, int((~good).sum()), got.ids[~good][:5].tolist(), behind[~good][:5].tolist())
        assert bool((got.ids == behind).any())


@pytest.mark.parametrize("n", [250, 1500])
def test_top_p_within_a_rounding_of_a_border(n, gpu):
    """Rows whose border by top-p lies between 1,500 likely tokens and unlikely ones a gap
    below, with the row's mass tuned so that p times it is those tokens' own mass up to a few
    roundings: the support is the likely tokens, or one more."""
    rng = np.random.default_rng(n)
    p, k, v = float(np.float32(0.9)), 1500, 6000
    z = np.full((n, v), -np.inf, np.float32)
    for row in range(n):
        head = -rng.random(k).astype(np.float32)
        head[0] = 0.0
        mass = math.fsum(np.exp(head.astype(np.float64)))
        tail = (-2.2 + 0.2 * rng.random(700)).astype(np.float32)
        left = mass / p * (1 + rng.integers(-8, 9) * 2.0 ** -53) - mass - math.fsum(np.exp(tail.astype(np.float64)))
        more = []
        while left > 1e-17 * mass and len(more) < 1500:
            x = np.float32(min(-2.05, math.log(left)))
            if math.exp(x) > left:
                x = np.nextafter(x, np.float32(-np.inf))
            more.append(x)
            left -= math.exp(x)
        assert len(more) < 1500
        every = np.concatenate([head, tail, np.array(more, np.float32)])
        z[row, rng.permutation(v)[:every.size]] = every
    z = torch.from_numpy(z).cuda()
    u = uniforms(n, 1)
    got = T.sample_tokens(z, u, top_p=0.9)
    w = z.double().exp()
    likely = z >= -1.0
    next_one = torch.where(likely, -math.inf, z).argmax(1, keepdim=True)
    good = torch.zeros(n, dtype=torch.bool, device="cuda")
    for keep in (likely, likely.scatter(1, next_one, True)):
        run = torch.where(keep, w, 0.0).cumsum(1)
        at = (run <= u[:, None] * run[:, -1:]).sum(1).int()
        one = got.ids == at
        logq = (w.gather(1, at.long()[:, None])[:, 0] / run[:, -1]).log()
        good |= one & ((got.logq.double() - logq).abs() <= 1e-6)
    assert bool(good.all()), (int((~good).sum()), got.ids[~good][:5].tolist())


@pytest.mark.parametrize("heat", [1.0, 0.5, 64.0])
def test_random_numbers_close_to_a_border_between_segments(heat, gpu):
    """Two tokens, in segments of their own, whose logits over the temperature are so large
    that their products with the rate are rounded by up to 6e-14: a random number 1e-14 on
    either side of the border between them, which is computed to 50 digits."""
    rate = 1.4426950408889634074 / heat
    lost = lambda m: Fraction(-(m * rate)) + Fraction(m) * Fraction(rate)  # noqa: E731
    rows, u, want = [], [], []
    for low in (600, 640, 680, -700):
        z = [torch.tensor((low + i * 0.013) * heat, dtype=torch.float32).item() for i in range(60)]
        z.sort(key=lost)
        for a, b in ((z[0], z[-1]), (z[-1], z[0]), (z[1], z[-2])):
            with decimal.localcontext() as c:
                c.prec = 50
                border = 1 / (1 + ((Decimal(b) - Decimal(a)) / Decimal(heat)).exp())
            for off, at in ((-1e-14, 1000), (1e-14, 3000)):
                rows.append((a, b))
                u.append(float(border + Decimal(off)))
                want.append(at)
    logit = torch.full((len(rows), 4096), -math.inf, device="cuda")
    logit[:, 1000], logit[:, 3000] = torch.tensor(rows, device="cuda").t()
    got = T.sample_tokens(logit, torch.tensor(u, dtype=torch.float64, device="cuda"), temperature=heat)
    assert got.ids.tolist() == want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_log_probabilities_to_their_rounding(dtype, gpu):
    """log q is computed in 64 bits throughout and rounded once: 2^-24 of itself.  So is
    log p where the row's mass at temperature 1 is that of all its tokens; otherwise its sum is
    made of 32-bit exponentials, off by 2^-23 and by 2^-24 for their correction, which are
    added in 64 bits.  (The logits are multiples of 1/8, so that their differences are exact;
    2^-40 stands for the 64-bit sums on either side.)"""
    n, v = 30, 60001
    z = (torch.randn((n, v), generator=gen(9), device="cuda") * 16).round().clamp(-64, 64) / 8
    z[:10] = z[:10].clamp(max=0.125)
    z[:, 77] += 3.0
    z = z.to(DT[dtype])
    u = uniforms(n, 9)
    for kw in FILTERS + [dict(top_k=2000), dict(top_p=0.8, temperature=0.9), dict(min_p=0.2, temperature=2.0)]:
        got = T.sample_tokens(z, u, **kw)
        ids, logq, logp = reference(z, u, **kw)
        assert torch.equal(got.ids, ids), kw
        exact = 2.0 ** -24 * logq.abs() + 2.0 ** -40
        assert bool(((got.logq.double() - logq).abs() <= exact).all()), (kw, "logq")
        plain = not kw or (list(kw) == ["top_p"])
        bound = 2.0 ** -24 * logp.abs() + 2.0 ** -40 + (0.0 if plain else 3 * 2.0 ** -24)
        assert bool(((got.logp.double() - logp).abs() <= bound).all()), (kw, "logp")


@pytest.mark.parametrize("n", [6, 300])
def test_min_p_where_weights_are_equal_in_64_bits(n, gpu):
    """At these temperatures every weight is 1 in double, and min-p 1 keeps them all, however
    many they are and with top-k as without."""
    for v in (100, 1000, 5000, 60000):
        z = logits(n, v, "f32", v)
        z[:, ::7] = -math.inf
        for heat in (1e20, 1e36):
            for kw in (dict(), dict(top_k=60), dict(top_k=2000)):
                check(z, uniforms(n, 1), temperature=heat, min_p=1.0, **kw)
