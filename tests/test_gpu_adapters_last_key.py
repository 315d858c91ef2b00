"""Adapters whose matrices are the last keys of the server, with ranks that are no multiple of eight, so many rows that matrices are laid: the shared matrix, A and B
and nothing behind, in either order.  Tolerances as in test_gpu_adapters.py."""
import numpy as np
import pytest

from test_gpu_adapters import _forward, _off
from test_gpu_experts import _close, _randn, _server, _type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,adapters,rank,rows,dim", [(8200, 16, 4, 1024, 1024), (13000, 5, 33, 72, 1000), (13000, 20, 20, 1000, 72), (13000, 5, 1, 1000, 200), (7000, 3, 7, 1024, 264)])
def test_last_keys(kind, n, adapters, rank, rows, dim):
    import torch
    L, W = max(rows, dim), adapters * rank
    rng = np.random.default_rng(n + rank)
    ids = rng.integers(0, adapters, size=n)
    ids[rng.random(n) < 0.1] = -1
    ids[-1] = adapters - 1
    x, dout = _randn(1, n, dim, kind=kind), _randn(2, n, rows, kind=kind, scale=0.1)
    for first_a, first_b in ((rows, rows + W), (rows + W, rows)):
        print("case", kind, n, adapters, rank, rows, dim, first_a, first_b, flush=True)
        srv, values = _server(rows + 2 * W, L, seed=rank, scale=0.1)
        w = values[:rows, :dim].double()
        a = values[first_a:first_a + W, :dim].reshape(adapters, rank, dim).double()
        b = values[first_b:first_b + W, :rows].reshape(adapters, rank, rows).double()
        groups = srv.group_rows(torch.from_numpy(ids).cuda(), adapters, pad=-1)
        out = srv.adapter_matmul(x.cuda(), groups, 0, rows, first_a, first_b, rank, dim=dim)
        dx, da, db = srv.adapter_grad(x.cuda(), dout.cuda(), groups, 0, first_a, first_b, rank)
        for got, given, (m, p, q), cols in ((out, x, (w, a, b), dim), (dx, dout, (w.t().contiguous(), b, a), rows)):
            want, s1, s2 = _forward(given, m, p, q, ids, 1.0)
            one = _off(kind, False, cols + rank)
            small = 4 * 2.0 ** -25 * (1 + given.double().abs().sum(1).max().item() * (1 + rank * float(q.abs().max()))) if kind == "float16" else 0.0
            _close(got, want, s1 * one + s2 * 3.1 * one, 1.0, kind, small)
        for e in range(adapters):
            p = torch.from_numpy(np.nonzero(ids == e)[0])
            for got, left, right, m in ((da[e], dout.double(), x.double(), b[e]), (db[e], x.double(), dout.double(), a[e])):
                low, mag = left[p] @ m.t(), left[p].abs() @ m.abs().t()
                _close(got, low.t() @ right[p], mag.t() @ right[p].abs(), (len(p) + max(rows, dim) + 60) * 2.0 ** -23, "float32")
        srv.status()
