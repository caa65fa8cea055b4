"""The operators around the logits on either side of the rules that choose a kernel's
form: what a wave carries from row to row, widths that fill three packs a lane, batches
in which every workgroup takes several rows, joins of many candidates.

Tolerances are those of test_gpu_logprobs.py and test_gpu_norm.py, whose checks are used;
bits are compared where the form must not change them."""
import math

import pytest
import torch

import test_gpu_logprobs as lp
import test_gpu_norm as norm
from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [20000, 20003])
def test_rows_beside_rows_with_forbidden_tokens(v, dtype, gpu):
    """Every workgroup takes several rows: what a row with -inf leaves behind in a wave
    changes no bit of the ones after it."""
    n = 3000
    fill = lp.normal(n, v, 1) * 3.0
    plain = lp.matrix(n, v, dtype, fill=fill)
    ids = lp.some_ids(n, v, 1)
    a = T.token_logprobs(plain, ids, k=20)
    fill[::3, ::7] = -math.inf
    fill[::97] = -math.inf  # and empty rows
    mixed = lp.matrix(n, v, dtype, fill=fill)
    b = T.token_logprobs(mixed, ids, k=20)
    same = torch.ones(n, dtype=torch.bool, device="cuda")
    same[::3] = False
    same[::97] = False
    for x, y in zip(a, b):
        assert torch.equal(x[same], y[same])
    some = torch.arange(0, n, 41, device="cuda")
    lp.check(lp.matrix(some.numel(), v, dtype, fill=fill[some]), ids[some].contiguous(), 20)
    assert bool((b.log_z[::97, 1] == 0).all()) and bool((b.entropy[::97] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,v,k", [(1, 151936, 96), (1, 1000000, 128), (1, 1500001, 3), (9, 400000, 128),
                                   (100, 33001, 128), (383, 9001, 11), (384, 9001, 11), (768, 8300, 60),
                                   (769, 8300, 60)])
def test_joins(n, v, k, dtype, gpu):
    """One chunk to several hundred, few candidates to tens of thousands."""
    lp.check(lp.matrix(n, v, dtype, fill=lp.normal(n, v, n + k)), lp.some_ids(n, v, k), k)


@pytest.mark.parametrize("k", [1, 50, 128])
def test_join_of_chunks_whose_best_lie_in_one(k, gpu):
    v = 151936
    fill = lp.normal(2, v, k)
    fill[0, 70000:70000 + 3 * k] += 40.0
    fill[1, :k] += 40.0
    lp.check(lp.matrix(2, v, "bf16", fill=fill), lp.some_ids(2, v, k), k)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 1025), ("bf16", 1032), ("bf16", 1200), ("bf16", 1536),
                                     ("f32", 516), ("f32", 768), ("f32", 767), ("f32", 772)])
def test_three_packs_a_lane(d, dtype, rms, gpu):
    w, b = norm.vectors(d, dtype, d)
    for n in (1, 6, 3001):
        x = norm.rows(n, d, dtype, d + n)
        norm.check_fwd(x, w, b, rms)
        norm.check_bwd(norm.rows(n, d, dtype, d + n + 1, shift=0.0), x, w, rms)


@pytest.mark.parametrize("dtype,n,d", [("bf16", 9000, 600), ("bf16", 9000, 680), ("bf16", 9000, 688),
                                       ("bf16", 2100, 2056), ("bf16", 2100, 2501), ("bf16", 1700, 3500),
                                       ("bf16", 1100, 3592), ("bf16", 1100, 4096), ("bf16", 700, 8200),
                                       ("bf16", 700, 16383), ("f32", 1700, 1537), ("f32", 700, 8193)])
def test_several_rows_a_workgroup(dtype, n, d, gpu):
    """Row sizes on both sides of the rule for the number of workgroups, each of which
    takes two rows or more."""
    w, _ = norm.vectors(d, "f32", d)
    x = norm.rows(n, d, dtype, d)
    norm.check_bwd(norm.rows(n, d, dtype, d + 1, shift=0.0), x, w, False)


def test_weights_that_are_not_numbers_stay_in_their_columns(gpu):
    """The elements of a pack that belong to its neighbour count for nothing, whatever
    they hold: only the output's and the gradient's own columns show a NaN weight."""
    n, d = 5, 1003
    w, b = norm.vectors(d, "bf16", d)
    w[d - 3] = math.nan
    x = norm.rows(n, d, "bf16", d)
    y, stats = T.norm_fwd(x, w, b)
    assert bool(torch.isnan(y[:, d - 3]).all()) and int(torch.isnan(y).sum()) == n
    gy = norm.rows(n, d, "bf16", d + 1, shift=0.0)
    _, gw, gb = T.norm_bwd(gy, x, w, stats, grad_bias=True)
    assert bool(torch.isfinite(gw).all()) and bool(torch.isfinite(gb).all())
