"""examples/head_step.py: the operators around the logits together, as a training
step and a served token use them."""
import importlib.util
import os

import pytest
import torch

from paper_2607_05804_amd import turnkl as T

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("head_step", os.path.join(ROOT, "examples", "head_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_loss_falls(example, gpu):
    losses = example.main(["--tokens", "301", "--hidden", "256", "--vocab", "5003", "--steps", "6",
                           "--topk", "20"])
    assert all(b < a for a, b in zip(losses, losses[1:])), losses


def test_a_steps_gradients_against_autograd(example, gpu):
    """The gradients that the step's calls give for the norm's weight and bias, against
    torch's autograd in 64 bits on the same inputs (alpha = 0: the trajectory mean).

    Tolerance: the logits and their gradient are rounded to bf16 on the way (2^-9 of each
    element, of mixed signs over 700 columns and 60 rows), so the sums are within a few
    2^-8 of their sizes: 5e-2 of the largest is ample."""
    n, d, v, k = 60, 64, 700, 10
    b = example.batch(n, d, v, 3, gpu)
    head = example.Head(d, v, n, k, 3)
    w0, b0, proj = head.weight.double(), head.bias.double(), head.proj.double()
    head.step(**b, alpha=0.0, policy=0.5, entropy=0.1, lr=0.0)

    w, bias = w0.clone().requires_grad_(), b0.clone().requires_grad_()
    x = b["hidden"].double()
    xc = x - x.mean(1, keepdim=True)
    z = (xc * (xc.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w + bias) @ proj.t()
    on = b["mask"] != 0
    ids = b["teacher_logits"].double().sort(dim=1, descending=True, stable=True).indices[:, :k]
    p, q = (t.gather(1, ids).log_softmax(1) for t in (z, b["teacher_logits"].double()))
    kl = (p.exp() * (p - q)).sum(1)
    trajs = [on & (b["traj"] == t) for t in b["traj"].unique()]
    trajs = [t for t in trajs if bool(t.any())]
    loss = sum(kl[t].mean() for t in trajs) / len(trajs)
    lp = z.log_softmax(1)
    h = -(lp.exp() * lp).sum(1)
    loss = loss - 0.5 / n * (b["advantage"].double() * lp.gather(1, b["sampled"].long()[:, None])[:, 0])[on].sum()
    loss = loss - 0.1 / n * h[on].sum()
    loss.backward()
    for got, ref in ((head.grad_w, w.grad), (head.grad_b, bias.grad)):
        assert float((got.double() - ref).abs().max()) <= 5e-2 * float(ref.abs().max())


def test_a_served_row(example, gpu):
    head = example.Head(128, 9001, 1, 5, 1)
    x = torch.randn(1, 128, device="cuda").bfloat16()
    ids, logp = head.serve(x, 5)
    z = head.logits(x)[2].double()
    ref = z.sort(dim=1, descending=True, stable=True).indices[0, :5]
    assert torch.equal(ids.long(), ref)
    assert bool(((logp.double() - z.log_softmax(1)[0, ref]).abs() <= 2e-5 + 1e-6 * 20).all())
