"""Ranks beyond 64, whose gradients go by other tiles, and as large as the sides.  Tolerances as in test_gpu_adapters.py."""
import numpy as np
import pytest

from test_gpu_adapters import _forward, _off
from test_gpu_experts import TYPES, _close, _randn, _server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,adapters,rank,rows,dim", [(70, 3, 65, 40, 24), (900, 4, 100, 130, 264), (3000, 2, 129, 200, 72), (13000, 3, 200, 72, 1000), (8200, 2, 300, 1024, 128), (2000, 40, 97, 128, 512)])
def test_large_ranks(kind, n, adapters, rank, rows, dim):
    import torch
    print("case", kind, n, adapters, rank, rows, dim, flush=True)
    L, W = max(rows, dim), adapters * rank
    rng = np.random.default_rng(n + rank)
    ids = rng.integers(0, adapters, size=n)
    ids[rng.random(n) < 0.1] = -1
    srv, values = _server(rows + 2 * W, L, seed=rank, scale=0.05)
    w, a, b = values[:rows, :dim].double(), values[rows:rows + W, :dim].reshape(adapters, rank, dim).double(), values[rows + W:, :rows].reshape(adapters, rank, rows).double()
    x, dout = _randn(1, n, dim, kind=kind), _randn(2, n, rows, kind=kind, scale=0.1)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), adapters, pad=-1)
    out = srv.adapter_matmul(x.cuda(), groups, 0, rows, rows, rows + W, rank, scale=0.5, dim=dim)
    dx, da, db = srv.adapter_grad(x.cuda(), dout.cuda(), groups, 0, rows, rows + W, rank, scale=0.5)
    for got, given, (m, p, q), cols in ((out, x, (w, a, b), dim), (dx, dout, (w.t().contiguous(), b, a), rows)):
        want, s1, s2 = _forward(given, m, p, q, ids, 0.5)
        one = _off(kind, kind == "float32", cols + rank)
        small = 4 * 2.0 ** -25 * (1 + given.double().abs().sum(1).max().item() * (1 + rank * float(q.abs().max()))) if kind == "float16" else 0.0
        _close(got, want, s1 * one + s2 * 3.1 * one, 1.0, kind, small)
    for e in range(adapters):
        p = torch.from_numpy(np.nonzero(ids == e)[0])
        for got, left, right, m in ((da[e], dout.double(), x.double(), b[e]), (db[e], x.double(), dout.double(), a[e])):
            low, mag = 0.5 * left[p] @ m.t(), 0.5 * left[p].abs() @ m.abs().t()
            _close(got, low.t() @ right[p], mag.t() @ right[p].abs(), (len(p) + max(rows, dim) + 60) * 2.0 ** -23, "float32")
    srv.status()
