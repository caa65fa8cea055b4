"""The token boundary of a model: from token ids to rows, between its blocks, and from
logits back to token ids, as a generation loop and as a training step.

The model is the smallest one in which every operator has its place: a table of token
rows, residual blocks whose branch is a gated two-layer product, and a projection onto
the vocabulary.  Its residual stream runs in fp32 beside bf16 products: embed_fwd
writes it from the bf16 table, and each block_norm_fwd adds a branch to it through the
block's gate and gives the next block's (at last the projection's) input.

  generate  embed_fwd -> [branch -> block_norm_fwd]* -> projection -> sample_tokens,
            the sampled ids being the next step's input, without a host round trip
  step      the same forward over whole sequences, token_logprobs and
            token_logprobs_bwd for the gradient of the logits, and back through
            [block_norm_bwd -> branch]* into the table's gradient by embed_bwd

  python examples/token_loop.py [--rows N] [--hidden D] [--vocab V] [--blocks B] [--tokens T]

Needs an MI355X.  Weights and prompts are random.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_05804_amd import turnkl as T  # noqa: E402

EPS = 1e-6


class Model:
    def __init__(self, hidden: int, vocab: int, blocks: int, *, wide: int = 0, seed: int = 0):
        dev = torch.device("cuda", torch.cuda.current_device())
        g = torch.Generator(device=dev).manual_seed(seed)
        wide = wide or 2 * hidden

        def rand(*shape, scale):
            return (torch.randn(*shape, generator=g, device=dev) * scale).bfloat16()

        self.hidden, self.vocab = hidden, vocab
        self.table = rand(vocab, hidden, scale=1.0)
        self.up = [rand(wide, hidden, scale=hidden ** -0.5) for _ in range(blocks)]
        self.down = [rand(hidden, wide, scale=wide ** -0.5) for _ in range(blocks)]
        # the norm in front of each block and, last, in front of the projection
        self.norm = [1 + 0.1 * torch.randn(hidden, generator=g, device=dev) for _ in range(blocks + 1)]
        self.gate = [0.5 + 0.1 * torch.randn(hidden, generator=g, device=dev) for _ in range(blocks)]
        self.proj = rand(vocab, hidden, scale=2.0 * hidden ** -0.5)

    def forward(self, ids, keep=None):
        """Logits of a batch of ids; `keep` collects what the backward pass reads."""
        h = T.embed_fwd(self.table, ids, dtype=torch.float32)
        y, stats = T.norm_fwd(h, self.norm[0], rms=True, eps=EPS)
        x = y.bfloat16()
        if keep is not None:
            keep.append((h, stats))
        for b, gate in enumerate(self.gate):
            u = x @ self.up[b].t()
            f = torch.relu(u) @ self.down[b].t()
            out = T.block_norm_fwd(h, f, self.norm[b + 1], gate=gate, rms=True, eps=EPS)
            if keep is not None:
                keep.append((x, u, f, out))
            h, stats, x = out.residual, out.stats, out.y
        return x @ self.proj.t(), x

    def gradients(self, ids, targets, mask=None):
        """Mean -log p of the targets and its gradients, by the names of the weights."""
        keep, g = [], {"norm": [None] * len(self.norm), "gate": [], "up": [], "down": []}
        z, x = self.forward(ids, keep)
        own = T.token_logprobs(z, targets, mask=mask, check=False)
        n = ids.numel() if mask is None else int(mask.sum())
        grad_z = T.token_logprobs_bwd(z, targets, own.log_z, own.entropy,
                                      grad_logp=torch.full_like(own.logp, -1.0 / max(n, 1)), mask=mask)
        loss = -own.logp.sum() / max(n, 1)
        g["proj"] = grad_z.t() @ x
        grad_y, grad_h = grad_z @ self.proj, None
        for b in reversed(range(len(self.gate))):
            x, u, f, out = keep[b + 1]
            grads = T.block_norm_bwd(grad_y, grad_h, out.residual, out.stats, f, self.norm[b + 1],
                                     gate=self.gate[b], rms=True)
            g["norm"][b + 1] = grads.weight
            g["gate"].insert(0, grads.gate)
            g["down"].insert(0, grads.branch.t() @ torch.relu(u))
            grad_u = (grads.branch @ self.down[b]) * (u > 0)
            g["up"].insert(0, grad_u.t() @ x)
            grad_y, grad_h = grad_u @ self.up[b], grads.residual
        h, stats = keep[0]
        grad_e, g["norm"][0], _ = T.norm_bwd(grad_y.float(), h, self.norm[0], stats, rms=True)
        if grad_h is not None:
            grad_e += grad_h
        g["table"] = torch.empty(self.vocab, self.hidden, device=h.device)
        T.embed_bwd(grad_e, ids, g["table"], mask=mask, check=False)
        return loss, g

    def generate(self, ids, tokens: int, u, *, temperature=0.8, top_k=50, top_p=0.95, workspace=None):
        """`tokens` further ids of each row, [tokens, n], with their log probabilities;
        u [tokens, n] in float64.  A row's ids stay on the GPU throughout."""
        steps, logp = [], []
        for t in range(tokens):
            z, _ = self.forward(ids)
            out = T.sample_tokens(z, u[t], temperature=temperature, top_k=top_k, top_p=top_p,
                                  workspace=workspace, check=False)
            ids = out.ids
            steps.append(ids)
            logp.append(out.logp)
        return torch.stack(steps), torch.stack(logp)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--rows", type=int, default=16)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=8)
    a = ap.parse_args(argv)
    m = Model(a.hidden, a.vocab, a.blocks)
    dev = m.table.device
    g = torch.Generator(device=dev).manual_seed(1)
    first = torch.randint(0, a.vocab, (a.rows,), generator=g, device=dev).int()
    u = torch.rand(a.tokens, a.rows, generator=g, device=dev, dtype=torch.float64)
    ids, logp = m.generate(first, a.tokens, u)
    for row in range(min(a.rows, 4)):
        print(f"row {row}:", ", ".join(f"{i} ({p:.2f})" for i, p in zip(ids[:, row].tolist(), logp[:, row].tolist())),
              flush=True)
    inputs = torch.cat([first[None], ids[:-1]]).reshape(-1)
    loss, _ = m.gradients(inputs, ids.reshape(-1))
    print(f"mean -log p of the generated tokens, before and after a step: {float(loss):.4f}, ", end="")
    loss, grads = m.gradients(inputs, ids.reshape(-1))
    m.proj -= (0.5 * grads["proj"].float()).to(m.proj.dtype)
    m.table -= (0.5 * grads["table"]).to(m.table.dtype)
    print(f"{float(m.gradients(inputs, ids.reshape(-1))[0]):.4f}")
    return ids


if __name__ == "__main__":
    main()
