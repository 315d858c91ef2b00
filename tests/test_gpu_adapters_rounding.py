"""Where rows and result have 16 bits, the low-rank numbers and both sides of the product that follows them are numbers of that type, whichever kernel takes a row: few
rows, tiles of several adapters, tiles of one, laid matrices.  Every result below is exact, so that a number that was not rounded shows."""
import pytest

pytestmark = pytest.mark.gpu

# n, adapters, columns of the result: one case at least for each kernel
CASES = [(5, 3, 40), (64, 200, 1024), (40, 2, 512), (500, 100, 200), (2000, 200, 1024), (600, 3, 200), (5000, 20, 1024), (13000, 5, 1000)]


def _filled(kind, adapters, columns):
    """Rows of 64 numbers, x, and W, A, B for results of so many columns.  u: a quarter of the step behind 1."""
    import torch
    u = torch.finfo(kind).eps / 4
    x, w = torch.zeros(64), torch.zeros(columns, 64)
    a, b = torch.zeros(adapters, 3, 64), torch.zeros(adapters, 3, columns)
    x[:8] = 1.0
    a[:, 0, 0], a[:, 0, 1], b[:, 0], w[:, 2] = 1.0, u, 1.0, -1.0                 # the low-rank number 1 + u is 1
    a[:, 1, 3], b[:, 1], w[:, 4] = 1.0, 1.0 + u, -1.0                            # B's number 1 + u is 1
    w[:, 5], w[:, 6] = 1.0 + u, -1.0                                            # and so is W's
    return x, w, a, b


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("n,adapters,columns", CASES)
def test_numbers_are_rounded_in_every_kernel(kind, n, adapters, columns):
    import torch
    from paper_2002_00655_amd import ps as P
    print("case", kind, n, adapters, columns, flush=True)
    kind = getattr(torch, kind)
    x, w, a, b = _filled(kind, adapters, columns)
    W, L = 3 * adapters, 1024
    for grad in (False, True):
        # the gradient of the rows: W and A, B turned round (rows of 64 come in, of `columns` go out)
        rows, dim = (64, columns) if grad else (columns, 64)
        values = torch.zeros(rows + 2 * W, L)
        values[:rows, :dim] = w.t() if grad else w
        values[rows:rows + W, :dim] = (b if grad else a).reshape(W, dim)
        values[rows + W:, :rows] = (a if grad else b).reshape(W, rows)
        srv = P.ParameterServer(values.shape[0], L, 1)
        srv.push(torch.arange(values.shape[0], device="cuda"), values.cuda())
        ids = torch.arange(n, device="cuda") * 7 % adapters
        groups = srv.group_rows(ids, adapters)
        given = x.to(kind).cuda().repeat(n, 1)
        if grad:
            call = lambda t: srv.adapter_grad(torch.zeros(n, dim, dtype=kind, device="cuda"), t, groups, 0, rows, rows + W, 3)[0]
        else:
            call = lambda t: srv.adapter_matmul(t, groups, 0, rows, rows, rows + W, 3, dim=dim)
        assert (call(given) == 0).all(), grad
        if kind == torch.float16:
            # a low-rank number beyond the type's largest is infinite, also where the product with B would bring it back
            more = torch.zeros(values.shape[0], L)
            more[rows + 2 + (W if grad else 0):rows + (2 * W if grad else W):3, 8] = 4.0
            more[rows + 2 + (0 if grad else W):rows + (W if grad else 2 * W):3, :columns] = 2.0 ** -10
            srv.push(torch.arange(values.shape[0], device="cuda"), more.cuda())
            assert (call(given) == 0).all(), grad
            given[:, 8] = 32768.0
            assert torch.isinf(call(given)).all(), grad
        srv.status()
