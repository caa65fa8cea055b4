"""A training step of a model's output end under distillation, with every operator
of the library that lies around the logits.

Frozen teacher: its hidden rows go through its projection, and token_logprobs takes
the teacher's top-K support with its log probabilities.  Student: its hidden rows go
through a norm (norm_fwd) and its projection; fwd_bwd_topk gives the distillation
loss and the gradient of the logits on that support; token_logprobs and
token_logprobs_bwd add a policy term, advantage times the sampled tokens' log
probabilities, and an entropy bonus; the gradient goes back through the projection
(a plain matrix product) and the norm (norm_bwd), and SGD updates the projection, the
norm's weight and bias.  Afterwards one new token is served: norm, projection, log
probabilities and alternatives of a single row.

  python examples/head_step.py [--tokens N] [--hidden D] [--vocab V] [--steps S]

Needs an MI355X.  Inputs are random; the loss falls because the student's hidden rows
and the teacher's are the same.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_05804_amd import turnkl as T  # noqa: E402


class Head:
    """Norm and projection of a student, with the buffers a step needs."""

    def __init__(self, hidden: int, vocab: int, tokens: int, k: int, turns: int):
        dev = torch.device("cuda", torch.cuda.current_device())
        bf16 = torch.bfloat16
        self.weight = torch.ones(hidden, device=dev)
        self.bias = torch.zeros(hidden, device=dev)
        self.proj = (torch.randn(vocab, hidden, device=dev) / hidden ** 0.5).to(bf16)
        self.grad_w, self.grad_b = torch.zeros_like(self.weight), torch.zeros_like(self.bias)
        self.norm_ws = T.NormWorkspace(tokens, hidden, device=dev)
        self.lp_ws = T.LogprobsWorkspace(tokens, vocab, k, device=dev)
        self.topk_ws = T.TopkWorkspace(tokens, k, turns, device=dev)
        self.k, self.turns = k, turns

    def logits(self, hidden):
        y, stats = T.norm_fwd(hidden, self.weight, self.bias)
        return y, stats, y @ self.proj.t()

    def step(self, hidden, teacher_logits, sampled, advantage, turn, traj, mask, *, alpha, policy,
             entropy, lr):
        """One SGD step; returns (distillation loss, mean log p of the sampled tokens,
        mean entropy) as device tensors."""
        n = hidden.shape[0]
        support = T.token_logprobs(teacher_logits, k=self.k, mask=mask, workspace=self.lp_ws,
                                   check=False)
        y, stats, z = self.logits(hidden)
        loss, grad, _, _, _, _ = T.fwd_bwd_topk(
            z, support.top_ids, support.top_logp, turn, traj, mask, alpha, max_turns=self.turns,
            workspace=self.topk_ws, check=False)
        # the loss falls as the policy term's log probabilities and the entropies rise
        own = T.token_logprobs(z, sampled, mask=mask, check=False)
        extra = T.token_logprobs_bwd(z, sampled, own.log_z, own.entropy,
                                     grad_logp=advantage * (-policy / n),
                                     grad_entropy=torch.full_like(advantage, -entropy / n),
                                     mask=mask, grad="inplace")  # the logits are not needed again
        grad += extra
        grad_y = grad @ self.proj
        T.norm_bwd(grad_y, hidden, self.weight, stats, grad_x=None, grad_weight=self.grad_w,
                   grad_bias=self.grad_b, workspace=self.norm_ws)
        self.proj -= (lr * (grad.t() @ y).float()).to(self.proj.dtype)
        self.weight -= lr * self.grad_w
        self.bias -= lr * self.grad_b
        asked = mask.sum().clamp(min=1)
        return loss[0], own.logp.sum() / asked, own.entropy.sum() / asked

    def serve(self, hidden, alternatives: int):
        """Greedy token of one row, its log probability and its alternatives."""
        _, _, z = self.logits(hidden)
        out = T.token_logprobs(z, k=alternatives, check=False)
        return out.top_ids[0], out.top_logp[0]


def batch(tokens, hidden, vocab, turns, device):
    g = torch.Generator(device=device).manual_seed(1)
    x = torch.randn(tokens, hidden, generator=g, device=device).bfloat16()
    teacher = (torch.randn(vocab, hidden, generator=g, device=device) * (3.0 / hidden ** 0.5)).bfloat16()
    per = max(1, -(-tokens // (2 * turns)))  # two trajectories of `turns` turns
    at = torch.arange(tokens, device=device)
    traj, turn = at // (per * turns), at // per % turns
    return {"hidden": x, "teacher_logits": x @ teacher.t(),
            "sampled": torch.randint(0, vocab, (tokens,), generator=g, device=device).int(),
            "advantage": torch.randn(tokens, generator=g, device=device),
            "turn": turn.int(), "traj": traj.int(), "mask": (at % per >= per // 3).to(torch.uint8)}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--tokens", type=int, default=1500)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--topk", type=int, default=50)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    dev = torch.device("cuda", torch.cuda.current_device())
    turns = 4
    b = batch(a.tokens, a.hidden, a.vocab, turns, dev)
    head = Head(a.hidden, a.vocab, a.tokens, a.topk, turns)
    losses = []
    for step in range(a.steps):
        loss, logp, entropy = head.step(**b, alpha=0.5, policy=0.01, entropy=0.001, lr=5.0)
        losses.append(float(loss))
        print(f"step {step}: top-{a.topk} KL {losses[-1]:.4f}, log p of the sampled tokens "
              f"{float(logp):.3f}, entropy {float(entropy):.3f}", flush=True)
    ids, logp = head.serve(b["hidden"][:1], 5)
    print("served token:", ", ".join(f"{i} ({p:.2f})" for i, p in zip(ids.tolist(), logp.tolist())))
    return losses


if __name__ == "__main__":
    main()
