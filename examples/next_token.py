"""A small next-token model whose parameters all lie in one parameter server, trained with the calls for token models.

    python examples/next_token.py [--steps 200] [--dim 128] [--vocab 2000]

The server's keys, each with 2 * dim values:

    vocab keys   input embeddings    [embedding | AdaGrad accumulator]
    vocab keys   output embeddings   [embedding | AdaGrad accumulator]
    length keys  position embeddings [embedding | not used]
    4 * dim keys the rows of four dim x dim matrices of two residual layers [weight | momentum]

A step looks up the batch's tokens, scores the next token against sampled others, and updates every parameter by the rule that
suits it: the rows that were looked up by AdaGrad, the matrices by their orthogonalised momentum, the short table of
positions by its whole gradient, accumulated over two halves of the batch.  The sequences are synthetic: four in five
tokens follow from the one before by a fixed permutation.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2002_00655_amd.ps import ParameterServer  # noqa: E402

PAD = -1                                              # stands behind the end of a sequence


class Model:
    def __init__(self, vocab, dim, length, workers=1, seed=0):
        self.vocab, self.dim, self.length = vocab, dim, length
        self.first_out, self.first_pos = vocab, 2 * vocab
        self.first_matrix = self.first_pos + length
        keys = self.first_matrix + 4 * dim
        self.server = ParameterServer(keys, 2 * dim, workers)
        g = torch.Generator().manual_seed(seed)
        values = torch.zeros(keys, 2 * dim)
        values[:, :dim] = torch.randn(keys, dim, generator=g) * 0.02
        values[self.first_matrix:, :dim] *= 0.5 / (0.02 * dim ** 0.5)
        self.server.push(torch.arange(keys, device="cuda"), values.cuda())
        self.matrix_keys = torch.arange(self.first_matrix, keys, device="cuda")
        self.scale = dim ** 0.5

    def embed(self, tokens, positions):
        """The input of the layers: scaled token embeddings (zero for padding) and position embeddings, [batch, length, dim]."""
        s = self.server
        return (s.emb_lookup(tokens, num_tokens=self.vocab, dim=self.dim, scale=self.scale, pad_token=PAD),
                s.emb_lookup(positions, first_key=self.first_pos, num_tokens=self.length, dim=self.dim))

    def candidates(self, tokens):
        return self.server.emb_lookup(tokens, first_key=self.first_out, num_tokens=self.vocab, dim=self.dim)

    def matrices(self):
        return self.server.pull(self.matrix_keys)[:, :self.dim].reshape(4, self.dim, self.dim)

    @staticmethod
    def layers(x, w):
        for i in (0, 2):
            x = x + torch.relu(x @ w[i].t()) @ w[i + 1].t()
        return x


def loss_of(x, w, out, real):
    """Mean cross-entropy of the right candidate, the first, among all, over the positions that are not padding."""
    scores = (Model.layers(x, w).unsqueeze(-2) * out).sum(-1)
    return (torch.logsumexp(scores, -1) - scores[..., 0])[real].sum() / real.sum().clamp(min=1)


def step(model, tokens, targets, negatives, lr, matrix_lr, position_lr):
    """One training step on [batch, length] tokens; returns the loss (on the device)."""
    s, dim = model.server, model.dim
    positions = torch.arange(model.length, device="cuda", dtype=torch.int32).expand(tokens.shape).contiguous()
    cands = torch.cat([targets.unsqueeze(-1), negatives.expand(*targets.shape, -1)], -1).contiguous()
    w = model.matrices().requires_grad_()
    grad_pos, total, parts = None, 0.0, []
    for half in torch.arange(tokens.shape[0], device="cpu").chunk(2):
        a, b = int(half[0]), int(half[-1]) + 1
        emb, pos = model.embed(tokens[a:b], positions[a:b])
        out = model.candidates(cands[a:b])
        for t in (emb, pos, out):
            t.requires_grad_()
        loss = loss_of(emb + pos, w, out, tokens[a:b] != PAD) * ((b - a) / tokens.shape[0])
        loss.backward()
        total = total + loss.detach()
        # positions that hold padding have a gradient of zero; the others of both halves add up
        grad_pos = s.emb_grad(positions[a:b], pos.grad, model.length, grad=grad_pos, accumulate=grad_pos is not None)
        parts.append((emb.grad, out.grad))
    s.emb_adagrad_step(tokens, torch.cat([p[0] for p in parts]), lr, 1e-8, num_tokens=model.vocab, scale=model.scale, pad_token=PAD)
    s.emb_adagrad_step(cands, torch.cat([p[1] for p in parts]), lr, 1e-8, first_key=model.first_out, num_tokens=model.vocab)
    s.push(torch.arange(model.first_pos, model.first_pos + model.length, device="cuda"),
           torch.cat([-position_lr * grad_pos, torch.zeros_like(grad_pos)], 1))
    s.muon_step(model.first_matrix, w.grad, matrix_lr, weight_decay=0.01)
    return total


def batches(vocab, batch, length, negatives, seed):
    """Endless (tokens, targets, negatives); the end of some sequences is padding."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda hi, *shape: torch.randint(0, hi, shape, device="cuda", generator=g)  # noqa: E731
    follow = torch.randperm(vocab, device="cuda", generator=g)
    while True:
        seq = [rand(vocab, batch)]
        for _ in range(length):
            seq.append(torch.where(torch.rand(batch, device="cuda", generator=g) < 0.8, follow[seq[-1]], rand(vocab, batch)))
        seq = torch.stack(seq, 1)
        tokens, targets = seq[:, :-1].contiguous(), seq[:, 1:].contiguous()
        behind = torch.arange(length, device="cuda") >= (length - rand(length // 2, batch).clamp(max=length // 4))[:, None]
        yield tokens.masked_fill(behind, PAD), targets, rand(vocab, negatives)


def train(steps=200, vocab=2000, dim=128, length=32, batch=64, negatives=63, lr=0.1, matrix_lr=0.01, position_lr=0.1, seed=0, report=None):
    model, data, losses = Model(vocab, dim, length, seed=seed), batches(vocab, batch, length, negatives, seed), []
    for i in range(steps):
        losses.append(step(model, *next(data), lr, matrix_lr, position_lr))
        if report and (i % 20 == 0 or i == steps - 1):
            report(i, float(losses[-1]))
    model.server.status()
    return model, [float(x) for x in losses]


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--vocab", type=int, default=2000)
    p.add_argument("--dim", type=int, default=128)
    p.add_argument("--batch", type=int, default=64)
    a = p.parse_args()
    train(a.steps, a.vocab, a.dim, batch=a.batch, report=lambda i, loss: print(f"step {i:5d}  loss {loss:.4f}", flush=True))


if __name__ == "__main__":
    main()
