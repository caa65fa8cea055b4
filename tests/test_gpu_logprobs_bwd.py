"""turnkl_token_logprobs_bwd against its formula in 64 bits and against central
differences of the forward definition.

Tolerances.  With y = log p in float (error at most 2^-23 (|z - M| + L), which
times p is below 2e-6 relative where p matters), p carries that, an ulp of exp2
and one of the product; G = gl [v = t] - p (gl + gh (y + H)) a few more.  For fp32
output |dG| <= 1e-5 (|p gl| + |p gh (log p + H)| + |gl [v = t]|) + 1e-30; bf16 adds
the rounding of the result, 2^-9 |G| (2^-8 taken), and its smallest normals.
"""
import math

import pytest
import torch

from paper_2607_05804_amd import turnkl as T
from test_gpu_logprobs import matrix, normal, pattern, some_ids

pytestmark = pytest.mark.gpu


def formula(z, ids, gl, gh, mask=None):
    """(G, sum of its terms' sizes) in float64."""
    z = z.double()
    n, v = z.shape
    gl = torch.zeros(n, device="cuda") if gl is None else gl
    gh = torch.zeros(n, device="cuda") if gh is None else gh
    gl, gh = gl.double()[:, None], gh.double()[:, None]
    lp = z.log_softmax(1)
    p = lp.exp()
    lp = torch.where(p > 0, lp, 0.0)
    h = -(p * lp).sum(1, keepdim=True)
    one = torch.zeros_like(z)
    if ids is not None:
        ok = ((ids >= 0) & (ids < v))[:, None]
        one.scatter_(1, torch.where(ok, ids[:, None], 0).long(), ok.double())
    g = gl * (one - p) - gh * p * (lp + h)
    size = (gl * one).abs() + (gl * p).abs() + (gh * p).abs() * (lp.abs() + h)
    off = (z.max(1, keepdim=True).values == -math.inf)
    if mask is not None:
        off = off | (mask == 0)[:, None]
    return torch.where(off, 0.0, g), torch.where(off, 0.0, size)


def check(z, ids, gl, gh, mask=None, grad="new"):
    out = T.token_logprobs(z, ids, mask=mask, check=False)
    ref, size = formula(z, ids, gl, gh, mask)
    got = T.token_logprobs_bwd(z, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh,
                               mask=mask, grad=grad)
    bound = 1e-5 * size + 1e-30
    if z.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs() + 2.0 ** -126
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bool(bad.any()), (bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), ref[bad][:5].tolist())
    return got


def upstream(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 3, 5, 7, 8, 9, 64, 127, 1000, 1024, 4095, 8191, 8192, 8193, 8200,
                               32000, 50257, 151936, 200001])
def test_vocabularies(v, dtype, gpu):
    z = matrix(6, v, dtype, fill=normal(6, v, v))
    gl, gh = upstream(6, v)
    ids = some_ids(6, v, v)
    check(z, ids, gl, gh)
    check(z, ids, gl, None)
    check(z, None, None, gh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v,pad,start", [(1000, 1, 0), (1000, 24, 1), (1003, 5, 3), (8200, 0, 7),
                                         (50257, 47, 0), (33, 3, 1), (6, 2, 1), (1, 3, 1)])
def test_starts_strides_and_padding(v, pad, start, dtype, gpu):
    """Columns between the rows of the gradient stay as they were; the logits and
    the gradient may start anywhere, apart from each other."""
    n = 5
    gl, gh = upstream(n, v)
    ids = some_ids(n, v, v)
    for lp, ls in ((pad, start), (0, 0), (3, 2)):
        z = matrix(n, v, dtype, lp, ls, normal(n, v, v))
        buf = torch.full((start + n * (v + pad) + 8,), 7.0, dtype=z.dtype, device="cuda")
        grad = buf[start:start + n * (v + pad)].view(n, v + pad)[:, :v]
        check(z, ids, gl, gh, grad=grad)
        rest = buf.clone()
        rest[start:start + n * (v + pad)].view(n, v + pad)[:, :v] = 7.0
        assert bool((rest == 7.0).all())
        # in place, also where packs are moved inside the row
        fresh = check(z, ids, gl, gh)
        out = T.token_logprobs(z, ids)
        T.token_logprobs_bwd(z, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh,
                             grad="inplace")
        assert torch.equal(z, fresh)


@pytest.mark.parametrize("name", ["constant", "peaked", "few_allowed", "one_allowed", "lowest",
                                  "all_lowest", "far", "spread", "late"])
def test_patterns(name, gpu):
    for dtype in ("bf16", "f32"):
        for n, v in ((4, 3001), (2, 32000)):
            z = matrix(n, v, dtype, fill=pattern(name, n, v))
            gl, gh = upstream(n, 3)
            check(z, some_ids(n, v, 2), gl, gh)


def test_masked_empty_and_undefined_rows(gpu):
    for v in (7, 3000, 50257):
        for dtype in ("bf16", "f32"):
            z = matrix(6, v, dtype, fill=normal(6, v, 1))
            z[1] = -math.inf
            z[3] = math.nan  # masked: not read
            mask = torch.tensor([1, 1, 1, 0, 1, 0], dtype=torch.uint8, device="cuda")
            gl, gh = upstream(6, 5)
            ids = some_ids(6, v, 1)
            got = T.token_logprobs_bwd(z, ids, *T.token_logprobs(z, ids, mask=mask)[2:0:-1],
                                       grad_logp=gl, grad_entropy=gh, mask=mask)
            assert bool((got[[1, 3, 5]] == 0).all())
            keep = [0, 2, 4]
            ref, size = formula(z[keep], ids[keep], gl[keep], gh[keep])
            tol = 1e-5 * size + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 0) + 1e-30
            assert bool(((got[keep].double() - ref).abs() <= tol + 2.0 ** -126).all())
            z[0, 0] = math.nan
            z[2, v - 1] = math.inf
            out = T.token_logprobs(z, ids, mask=mask)
            got = T.token_logprobs_bwd(z, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh,
                                       mask=mask)
            assert bool(got[0].isnan().all()) and bool(got[2].isnan().all())
            assert not bool(got[4].isnan().any())


def test_ids_out_of_range_have_no_column(gpu):
    n, v = 4, 1000
    z = matrix(n, v, "f32", fill=normal(n, v, 1))
    ids = torch.tensor([-1, v, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    gl, gh = upstream(n, 2)
    check(z, ids, gl, gh)


def test_central_differences(gpu):
    """The gradient against differences of logp and H as their definitions give
    them in 64 bits: the formula itself is right."""
    n, v = 3, 40
    z = normal(n, v, 4).double()
    ids = some_ids(n, v, 4)
    gl, gh = upstream(n, 6)

    def value(a):
        lp = a.log_softmax(1)
        h = -(lp.exp() * lp).sum(1)
        return gl.double() * lp.gather(1, ids.long()[:, None])[:, 0] + gh.double() * h

    step = 1e-5
    ref = torch.empty_like(z)
    for c in range(v):
        d = torch.zeros_like(z)
        d[:, c] = step
        ref[:, c] = (value(z + d) - value(z - d)) / (2 * step)
    zf = z.float()
    out = T.token_logprobs(zf, ids)
    got = T.token_logprobs_bwd(zf, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh)
    # differences of rounded 64-bit values: 1e-16 / 1e-5 times the values; z.float() moves z by 2^-24 |z|
    assert bool(((got.double() - ref).abs() <= 2e-6 * (1 + ref.abs())).all())


def test_offsets_past_32_bits(gpu):
    n, v = 30000, 151936
    z = torch.zeros((n, v), dtype=torch.bfloat16, device="cuda")
    z[-3:] = normal(3, v, 6).to(torch.bfloat16)
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[-3:] = some_ids(3, v, 6)
    gl, gh = upstream(n, 1)
    out = T.token_logprobs(z, ids)
    small = T.token_logprobs_bwd(z[-3:].clone(), ids[-3:].clone(), out.log_z[-3:].clone(),
                                 out.entropy[-3:].clone(), grad_logp=gl[-3:].clone(),
                                 grad_entropy=gh[-3:].clone())
    T.token_logprobs_bwd(z, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh, grad="inplace")
    assert torch.equal(z[-3:], small)


def test_graph_replays_equal_eager(gpu):
    n, v = 50, 32001
    z = matrix(n, v, "bf16", fill=normal(n, v, 1))
    ids = some_ids(n, v, 1)
    gl, gh = upstream(n, 1)
    out, ws = T.new_token_logprobs(n), T.LogprobsWorkspace(n, v)
    grad = torch.empty_like(z)

    def step():
        T.token_logprobs(z, ids, out=out, workspace=ws, check=False)
        T.token_logprobs_bwd(z, ids, out.log_z, out.entropy, grad_logp=gl, grad_entropy=gh, grad=grad)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    for r in range(4):
        z.copy_(normal(n, v, 20 + r))
        grad.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        got = grad.clone()
        step()
        assert torch.equal(got.view(torch.int16), grad.view(torch.int16))


def test_binding_refuses(gpu):
    z = matrix(4, 100, "bf16", fill=normal(4, 100, 1))
    ids = some_ids(4, 100, 1)
    gl, gh = upstream(4, 1)
    o = T.token_logprobs(z, ids)
    with pytest.raises(T.TurnKLError):  # nothing to differentiate
        T.token_logprobs_bwd(z, ids, o.log_z, o.entropy)
    with pytest.raises(T.TurnKLError):
        T.token_logprobs_bwd(z, None, o.log_z, o.entropy, grad_logp=gl)
    with pytest.raises(T.TurnKLError):
        T.token_logprobs_bwd(z, ids, o.log_z, None, grad_entropy=gh)
    for kw in (dict(grad=torch.empty(4, 99, dtype=z.dtype, device="cuda")), dict(grad="old"),
               dict(grad=torch.empty(4, 100, device="cuda")), dict(grad_logp=gl[:3])):
        with pytest.raises(ValueError):
            T.token_logprobs_bwd(z, ids, o.log_z, o.entropy, **{"grad_logp": gl, **kw})
    with pytest.raises(TypeError):
        T.token_logprobs_bwd(z, ids, o.log_z, o.entropy, grad_logp=gl.double())
