"""The example that trains a next-token model with its parameters in one server: the loss falls, and one step changes the
server as the formulas in 64 bits do."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("next_token", os.path.join(ROOT, "examples", "next_token.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_loss_falls(example):
    _, losses = example.train(steps=60, vocab=500, dim=64, length=16, batch=32, negatives=31)
    first, last = np.mean(losses[:3]), np.mean(losses[-5:])
    print(f"  loss {first:.3f} -> {last:.3f}")
    assert abs(losses[0] - np.log(32)) < 0.5 and last < 0.75 * first              # (before the first step: all candidates alike)


def test_one_step_in_64_bits(example):
    """The same step by torch in 64 bits on the server's values; what is compared is a few roundings of values below 1."""
    import torch
    vocab, dim, length, batch = 60, 32, 6, 8
    m = example.Model(vocab, dim, length, seed=3)
    s, keys = m.server, torch.arange(m.server.K, device="cuda")
    before = s.pull(keys).double()
    tokens, targets, neg = next(example.batches(vocab, batch, length, 7, 1))
    example.step(m, tokens, targets, neg, 0.1, 0.02, 0.3)
    got = s.pull(keys).double()

    p = before[:, :dim].clone().requires_grad_()
    cands = torch.cat([targets.unsqueeze(-1), neg.expand(*targets.shape, -1)], -1)
    real = tokens != example.PAD
    x = torch.where(real[..., None], p[tokens.clamp(min=0)] * m.scale, torch.zeros((), dtype=torch.float64, device="cuda"))
    x = x + p[m.first_pos:m.first_pos + length]
    w = p[m.first_matrix:].reshape(4, dim, dim)
    total = sum(example.loss_of(x[a:b], w, p[m.first_out + cands[a:b]], real[a:b]) / 2 for a, b in ((0, batch // 2), (batch // 2, batch)))
    (g,) = torch.autograd.grad(total, p)
    want = before.clone()
    rows = slice(0, 2 * vocab)
    want[rows, dim:] += g[rows] ** 2
    want[rows, :dim] -= torch.where(g[rows] != 0, 0.1 * g[rows] / torch.sqrt(want[rows, dim:] + 1e-8), torch.zeros_like(g[rows]))
    pos = slice(m.first_pos, m.first_pos + length)
    want[pos, :dim] -= 0.3 * g[pos]
    for i in range(4):
        at = slice(m.first_matrix + i * dim, m.first_matrix + (i + 1) * dim)
        want[at, dim:] = g[at]                                                # the first momentum
        d = g[at] + 0.95 * g[at]
        y = d / (torch.linalg.vector_norm(d) + 1e-7)
        for _ in range(5):
            h = y @ y.t()
            y = 3.4445 * y + (-4.7750 * h + 2.0315 * h @ h) @ y
        want[at, :dim] = want[at, :dim] * (1 - 0.02 * 0.01) - 0.02 * y
    err = (got - want).abs()
    # the gradients are 32-bit sums of a few hundred products of numbers up to about 1: 1e-6 of the largest; AdaGrad's first step is
    # lr * sign(g) whatever g's size, with an error of lr * dg / |g| where |g| is small against that
    dg = 1e-6 * g.abs().max()
    first = 0.1 * torch.minimum(dg / g[rows].abs().clamp(min=1e-30), torch.full_like(g[rows], 2.0)) + 1e-6
    assert (err[rows, :dim] <= torch.where(g[rows] != 0, first, torch.full_like(first, 1e-12))).all()
    assert (err[rows, dim:] <= 2 * g[rows].abs() * dg + dg ** 2).all()
    assert (err[pos, :dim] <= 0.3 * dg + 1e-7).all() and (got[pos, dim:] == 0).all()
    assert (err[m.first_matrix:, dim:] <= dg).all()
    # the orthogonalised matrix passes a relative error of its gradient on up to 485-fold
    assert (torch.linalg.vector_norm(err[m.first_matrix:, :dim]) <= 0.02 * 485 * 1e-6 * 4 * dim ** 0.5).all()
