"""norm_bwd of parts of its outputs at every width: the same bits as with all of them, and
no kernel whose result nobody takes."""
import ctypes

import pytest
import torch

import test_gpu_norm as norm
from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu


def kernels_of(call):
    """How many nodes a call leaves in a captured graph (asked of the runtime that is
    loaded)."""
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64.so" in line)
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    call()
    with torch.cuda.graph(graph):
        call()
    n = ctypes.c_size_t(0)
    rc = ctypes.CDLL(path).hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(n))
    assert rc == 0
    return n.value


@pytest.mark.parametrize("dtype,d", [("f32", 9000), ("f32", 16384), ("f32", 8192), ("bf16", 9000)])
def test_sums_without_the_rows_gradient(dtype, d, gpu):
    n = 40
    x, gy = norm.rows(n, d, dtype, 1), norm.rows(n, d, dtype, 2)
    w, b = norm.vectors(d, "f32", 3)
    for rms in (False, True):
        stats = T.norm_fwd(x, w, b, rms=rms)[1]
        gx, gw, gb = T.norm_bwd(gy, x, w, stats, rms=rms, grad_bias=True)
        norm.check_bwd(gy, x, w, rms, grad_x=None)
        none, gw2, gb2 = T.norm_bwd(gy, x, w, stats, rms=rms, grad_x=None, grad_bias=True)
        assert none is None and torch.equal(gw, gw2) and torch.equal(gb, gb2)
        none, none2, gb2 = T.norm_bwd(gy, x, w, stats, rms=rms, grad_x=None, grad_weight=None, grad_bias=True)
        assert none is None and none2 is None and torch.equal(gb, gb2)
        alone = T.norm_bwd(gy, x, w, stats, rms=rms, grad_weight=None)
        assert torch.equal(alone[0], gx) and alone[1] is None


@pytest.mark.parametrize("dtype,d,kernels", [("f32", 9000, 2), ("f32", 8192, 2), ("bf16", 16384, 2)])
def test_sums_alone_take_two_kernels(dtype, d, kernels, gpu):
    """The sums and their join; the rows' gradient is not worked out for nobody."""
    x, gy = norm.rows(40, d, dtype, 1), norm.rows(40, d, dtype, 2)
    w, _ = norm.vectors(d, "f32", 3)
    stats = T.norm_fwd(x, w)[1]
    gw, ws = torch.empty(d, device="cuda"), T.NormWorkspace(40, d)
    assert kernels_of(lambda: T.norm_bwd(gy, x, w, stats, grad_x=None, grad_weight=gw,
                                         workspace=ws)) == kernels
