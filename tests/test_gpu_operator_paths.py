"""Token log probabilities on the paths that long rows take: what is reported of bad ids
by rows of one chunk and by the join of several, lists of the rows asked for, and rows of
which more elements reach the bound of the alternatives than the lists hold.  Checks and
tolerances are those of test_gpu_logprobs.py.

The statistics of the norm: their own errors.  A row's sum of squared differences errs by
60 u of itself (u = 2^-24: at most 32 terms a thread and a tree of 14, and the difference's
own rounding twice), the square of the mean's error, 60 u mean |x|, is added to it, and r
takes half of that relative to the variance, with a quotient, a root and a reciprocal of u
each: |dr| <= r (3e-6 + (60 u mean |x| r)^2)."""
import math

import pytest
import torch

import test_gpu_logprobs as lp
import test_gpu_norm as norm
from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


# one wave a row; rows of one chunk, one listed and one looked up; chunks that fill the
# card; chunks because of the row's size
@DTYPES
@pytest.mark.parametrize("n,v", [(70, 2000), (800, 20001), (500, 20000), (70, 50257), (1, 151936),
                                 (3, 200000), (780, 196700)])
def test_bad_ids(n, v, dtype, gpu):
    z = lp.matrix(n, v, dtype, fill=lp.normal(n, v, 3))
    at = sorted({n // 2, n - 1})
    for k in (0, 4):
        ws = T.LogprobsWorkspace(n, v, k)
        for bad in (-1, v, 2 ** 31 - 1, -2 ** 31):
            ids = lp.some_ids(n, v, 3)
            ids[at] = bad
            out = lp.check(z, ids, k, workspace=ws, check=False)
            assert out.logp[at].isnan().all() and ws.status() == T.ERR_TOKEN_ID
            with pytest.raises(T.TurnKLError, match="id outside"):
                T.token_logprobs(z, ids, k=k, workspace=ws)
            mask = torch.ones(n, dtype=torch.uint8, device="cuda")
            mask[at] = 0  # nobody asks for those rows: the same workspace, without an error
            lp.check(z, ids, k, mask, workspace=ws)
            assert ws.status() == T.OK
            ids[at] = 0
            T.token_logprobs(z, ids, k=k, workspace=ws)


@DTYPES
@pytest.mark.parametrize("n,v,k", [(767, 9001, 5), (768, 9001, 5), (1100, 20000, 50), (16383, 8300, 3),
                                   (16385, 8301, 3), (33000, 8304, 0), (780, 196700, 20)])
def test_scattered_masks(n, v, k, dtype, gpu):
    """Rows that are not asked for hold NaN and ids that do not exist."""
    if dtype == "f32":
        n = min(n, 16385)
    g = torch.Generator(device="cuda").manual_seed(n)
    fill = lp.normal(n, v, n)
    for share in (0.5, 0.03, 0.97):
        mask = (torch.rand(n, generator=g, device="cuda") < share).to(torch.uint8)
        mask[0], mask[-1] = share > 0.1, share < 0.9
        z = lp.matrix(n, v, dtype, fill=fill)
        z[mask == 0] = math.nan
        ids = lp.some_ids(n, v, n)
        ids[mask == 0] = -7
        step = 4000
        out = T.token_logprobs(z, ids, k=k, mask=mask)
        for r in range(0, n, step):
            part = slice(r, min(n, r + step))
            ref = lp.reference(z[part], ids[part], k, mask[part])
            lp.close(out.logp[part], ref["logp"], 2e-5, 1e-6, "logp")
            lp.close(out.entropy[part], ref["entropy"], 4e-5, 4e-5, "entropy")
            lp.close(out.log_z[part, 1], ref["L"], 2e-5, 1e-6, "L")
            lp.close(out.log_z[part, 0], ref["M"], 0.0, 0.0, "M")
            if k:
                assert torch.equal(out.top_ids[part], ref["top_ids"])
                lp.close(out.top_logp[part], ref["top_logp"], 2e-5, 1e-6, "top_logp")
    none = torch.zeros(n, dtype=torch.uint8, device="cuda")
    out = T.token_logprobs(z, ids, k=k, mask=none)
    assert not bool(out.logp.any()) and not bool(out.entropy.any()) and bool(out.log_z.isnan().all())
    if k:
        assert bool((out.top_ids == -1).all()) and bool((out.top_logp == -math.inf).all())


@DTYPES
@pytest.mark.parametrize("n,v,k", [(1, 151936, 20), (40, 50257, 128), (900, 20001, 20), (900, 20000, 1),
                                   (1500, 9001, 50), (300, 3001, 20)])
def test_more_candidates_than_the_lists_hold(n, v, k, dtype, gpu):
    """Rows in turn: ten allowed tokens; few values; a long run of equal largest ones; all
    forbidden; NaN or +inf beside ordinary ones; ordinary."""
    g = torch.Generator(device="cuda").manual_seed(v)
    z = lp.normal(n, v, v)
    allowed = torch.randint(0, v, (n, 10), generator=g, device="cuda")
    few = torch.full_like(z, -math.inf).scatter(1, allowed, z.gather(1, allowed))
    z[0::6] = few[0::6]
    z[1::6] = (z[1::6] * 0.3).round()
    z[2::6, v // 2:v // 2 + 1500] = 30.0
    z[3::6] = -math.inf
    z[4::6, v // 3] = math.nan
    z[4::12, v // 7] = math.inf
    z = lp.matrix(n, v, dtype, fill=z)
    ids = lp.some_ids(n, v, 1)
    first = lp.check(z, ids, k)
    for _ in range(3):
        for a, b in zip(first, T.token_logprobs(z, ids, k=k)):
            assert torch.equal(a.view(torch.int32), b.view(torch.int32))


@DTYPES
@pytest.mark.parametrize("d", [1, 3, 64, 1000, 1537, 4096, 8200, 16384])
def test_statistics_of_the_norm(d, dtype, gpu):
    for scale, shift, eps in ((1.0, 0.25, 1e-6), (1.0, 1000.0, 1e-6), (1e-12, 0.0, 0.0), (1e12, 0.0, 1e-6),
                              (1.0, 0.0, 100.0), (0.0, 2.5, 1e-6)):
        if d == 1 and eps == 0.0:
            continue  # a row without variance and eps has no r
        x = norm.rows(37, d, dtype, d, scale=scale, shift=shift)
        size = x.double().abs().mean(1, keepdim=True)
        for rms in (False, True):
            mu, r = norm.statistics(x, rms, eps)
            stats = T.norm_fwd(x, rms=rms, eps=eps)[1]
            norm.assert_close(stats[:, :1], mu, 0.0 * mu if rms else 60 * 2.0 ** -24 * size + 1e-30, "mu")
            mean_error = 0.0 if rms else 60 * 2.0 ** -24 * size * r
            norm.assert_close(stats[:, 1:], r, r * (3e-6 + mean_error ** 2), "r")
