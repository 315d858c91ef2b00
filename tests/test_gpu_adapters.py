"""A shared projection with a low-rank adapter per row, and its gradients, against the formulas in 64 bits.

Tolerances, element by element: with S1 the sum of the absolute values of W's terms and S2 that of the adapter's, numbers of the server are off by half a step of the
products' type (W, A and B), and so are the low-rank numbers where they are multiplied in 16 bits; sums of K terms by K + 8 units of 2^-23; the result by half a step
of its own type."""
import numpy as np
import pytest

from test_gpu_experts import HALF, TYPES, _close, _randn, _server, _type

pytestmark = pytest.mark.gpu

CASES = [
    # n, adapters, rank, rows, dim, L
    (1, 1, 1, 1, 1, 1),
    (1, 5, 16, 64, 128, 128),
    (7, 3, 5, 33, 127, 130),
    (64, 200, 16, 256, 200, 256),
    (150, 4, 8, 100, 51, 200),
    (700, 3, 20, 65, 264, 264),
    (1200, 90, 7, 130, 72, 130),
    (3000, 2, 33, 200, 136, 272),
    (5000, 7, 64, 512, 96, 512),
    (9000, 3, 4, 1000, 264, 1000),
    (13000, 20, 20, 1000, 72, 1000),                 # (W and B laid)
    (13000, 5, 33, 72, 1000, 1000),                  # (the same of the gradient)
]


def _setup(case, seed=0, spoil=False):
    import torch
    n, adapters, rank, rows, dim, L = case
    first, first_a = 2, 2 + rows + 1
    first_b = first_a + adapters * rank + 3
    srv, values = _server(first_b + adapters * rank + 1, L, seed=n + seed, scale=0.1)
    if spoil:
        bad = torch.zeros_like(values)
        bad[first:first + rows, dim:] = float("nan")
        bad[first_a:first_a + adapters * rank, dim:] = float("nan")
        bad[first_b:first_b + adapters * rank, rows:] = float("nan")
        for k in (0, 1, first + rows, first_b - 1, first_b - 2, first_b - 3, first_b + adapters * rank):
            bad[k] = float("inf")
        srv.push(torch.arange(values.shape[0], device="cuda"), bad.cuda())
    w = values[first:first + rows, :dim].double()
    a = values[first_a:first_a + adapters * rank, :dim].reshape(adapters, rank, dim).double()
    b = values[first_b:first_b + adapters * rank, :rows].reshape(adapters, rank, rows).double()
    rng = np.random.default_rng(n + seed)
    ids = np.sort(rng.integers(0, adapters, size=max(1, n // 20 + 1)))[rng.integers(0, max(1, n // 20 + 1), size=n)]
    ids[rng.random(n) < 0.15] = -1
    return srv, (first, first_a, first_b), w, a, b, ids


def _forward(x, w, a, b, ids, scale):
    """The result, and S1 and S2."""
    import torch
    x = x.double()
    out, s1, s2 = x @ w.t(), x.abs() @ w.abs().t(), torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64)
    for e in range(a.shape[0]):
        p = torch.from_numpy(np.nonzero(ids == e)[0])
        out[p] += scale * (x[p] @ a[e].t()) @ b[e]
        s2[p] = abs(scale) * (x[p].abs() @ a[e].abs().t()) @ b[e].abs()
    return out, s1, s2


def _off(kind, precise, K):
    return (K + 8) * 2.0 ** -23 + (0.0 if precise else HALF[kind] * (1 + 2.0 ** -9))


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("kind", TYPES)
def test_adapter_matmul(case, kind):
    import torch
    n, adapters, rank, rows, dim, L = case
    print("case", case, kind, flush=True)
    srv, (first, first_a, first_b), w, a, b, ids = _setup(case, spoil=True)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), adapters, pad=-1)
    x, scale = _randn(1, n, dim, kind=kind), 0.7
    want, s1, s2 = _forward(x, w, a, b, ids, scale)
    for out_kind in (kind, "float32"):
        out = srv.adapter_matmul(x.cuda(), groups, first, rows, first_a, first_b, rank, scale=scale, dim=dim, dtype=_type(out_kind))
        precise = "float32" in (kind, out_kind)
        one = _off(kind, precise, dim + rank)
        small = 4 * 2.0 ** -25 * (1 + x.double().abs().sum(1).max().item() * (1 + rank * float(b.abs().max()))) if kind == "float16" and not precise else 0.0
        _close(out, want, s1 * one + s2 * 3.1 * one, 1.0, out_kind, small)
    srv.status()


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("kind", TYPES)
def test_adapter_grad(case, kind):
    import torch
    n, adapters, rank, rows, dim, L = case
    print("case", case, kind, flush=True)
    srv, (first, first_a, first_b), w, a, b, ids = _setup(case, seed=1, spoil=True)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), adapters, pad=-1)
    x, dout, scale = _randn(2, n, dim, kind=kind), _randn(3, n, rows, kind=kind, scale=0.1), 0.6
    dx, da, db = srv.adapter_grad(x.cuda(), dout.cuda(), groups, first, first_a, first_b, rank, scale=scale)
    assert da.shape == a.shape and db.shape == b.shape and dx.dtype == x.dtype and da.dtype == db.dtype == torch.float32
    # dx is the same product with W, A and B turned round
    want, s1, s2 = _forward(dout, w.t().contiguous(), b, a, ids, scale)
    one = _off(kind, kind == "float32", rows + rank)
    small = 4 * 2.0 ** -25 * (1 + dout.double().abs().sum(1).max().item() * (1 + rank * float(a.abs().max()))) if kind == "float16" else 0.0
    _close(dx, want, s1 * one + s2 * 3.1 * one, 1.0, kind, small)
    xd, dd = x.double(), dout.double()
    for e in range(adapters):
        p = torch.from_numpy(np.nonzero(ids == e)[0])
        for got, left, right, m in ((da[e], dd, xd, b[e]), (db[e], xd, dd, a[e])):
            low, mag = scale * left[p] @ m.t(), abs(scale) * left[p].abs() @ m.abs().t()
            _close(got, low.t() @ right[p], mag.t() @ right[p].abs(), (len(p) + max(rows, dim) + 60) * 2.0 ** -23, "float32")
            if len(p) == 0:
                assert (got == 0).all()
    none, da2, db2 = srv.adapter_grad(x.cuda(), dout.cuda(), groups, first, first_a, first_b, rank, scale=scale, want_dx=False)
    assert none is None and torch.equal(da, da2) and torch.equal(db, db2)
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [40, 300, 2000, 9000, 26000])
def test_an_adapter_that_is_no_number_spoils_no_other(kind, n):
    """Infinities of one adapter's matrices, and rows that are no numbers: others in the same tile stay."""
    import torch
    case = (n, 6, 8, 512, 128, 512)
    srv, (first, first_a, first_b), w, a, b, ids = _setup(case)
    rows, dim, rank = 512, 128, 8
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), 6, pad=-1)
    x, dout = _randn(2, n, dim, kind=kind), _randn(3, n, rows, kind=kind)

    def results():
        return (srv.adapter_matmul(x.cuda(), groups, first, rows, first_a, first_b, rank, dim=dim).float(),
                *(t.float() for t in srv.adapter_grad(x.cuda(), dout.cuda(), groups, first, first_a, first_b, rank)))
    y, dx, da, db = results()
    bad = torch.zeros(srv.K, srv.L)
    bad[first_b + 2 * rank + 3, :rows] = float("inf")                   # adapter 2: a row of B transposed
    bad[first_a + 2 * rank + 1, 5] = float("nan")                       # ... and a number of A
    srv.push(torch.arange(srv.K, device="cuda"), bad.cuda())
    p = int(np.nonzero(ids == 4)[0][0])                                 # a row of adapter 4
    x[p, 0] = float("nan")
    y2, dx2, da2, db2 = results()
    others = torch.from_numpy((ids != 2) & (np.arange(n) != p)).cuda()
    assert torch.equal(y2[others], y[others]) and torch.isfinite(y2[others]).all()
    others[p] = True                                                    # (dx needs no x)
    assert torch.equal(dx2[others], dx[others]) and torch.isfinite(dx2[others]).all()
    keep = [0, 1, 3, 5]
    assert torch.equal(da2[keep], da[keep]) and torch.equal(db2[keep], db[keep])
    assert torch.isnan(y2[torch.from_numpy(ids == 2).cuda()]).all() and torch.isnan(y2[p]).all()
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
def test_strides_and_shapes(kind):
    import torch
    case = (600, 5, 12, 96, 72, 96)
    n, adapters, rank, rows, dim, L = case
    srv, (first, first_a, first_b), w, a, b, ids = _setup(case)
    groups = srv.group_rows(torch.from_numpy(ids.reshape(20, 30)).cuda(), adapters, pad=-1)
    x = _randn(4, n, dim, kind=kind).cuda()
    dout = _randn(5, n, rows, kind=kind).cuda()
    want = srv.adapter_matmul(x, groups, first, rows, first_a, first_b, rank, dim=dim)
    grads = srv.adapter_grad(x, dout, groups, first, first_a, first_b, rank)
    assert torch.equal(srv.adapter_matmul(x.view(20, 30, dim), groups, first, rows, first_a, first_b, rank, dim=dim), want.view(20, 30, rows))
    assert srv.adapter_grad(x.view(20, 30, dim), dout.view(20, 30, rows), groups, first, first_a, first_b, rank)[0].shape == (20, 30, dim)
    for before, gap in ((1, 0), (8, 8), (3, 2)):
        def framed(t):
            f = torch.full((n, before + t.shape[1] + gap), float("nan"), dtype=t.dtype, device="cuda")
            f[:, before:before + t.shape[1]].copy_(t)
            return f[:, before:before + t.shape[1]]
        to = torch.full((n, before + rows + gap), 7.0, dtype=_type(kind), device="cuda")
        out = srv.adapter_matmul(framed(x), groups, first, rows, first_a, first_b, rank, dim=dim, out=to[:, before:before + rows])
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert (to == 7.0).all()
        for got, known in zip(srv.adapter_grad(framed(x), framed(dout), groups, first, first_a, first_b, rank), grads):
            assert torch.equal(got, known)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [40, 700, 9000])
def test_orders_that_are_none_do_no_harm(kind, n):
    """As products with experts: numbers out of range are found where they are read, offsets that do not rise are nobody's rows."""
    import torch
    from paper_2002_00655_amd import ps as P
    adapters, rank, rows, dim = 3, 8, 1024, 64
    first_a, first_b = rows, rows + adapters * rank
    srv, _ = _server(first_b + adapters * rank, 1024, seed=n, scale=0.1)
    x, dout = _randn(1, n, dim, kind=kind).cuda(), _randn(2, n, rows, kind=kind).cuda()
    calls = (lambda g: srv.adapter_matmul(x, g, 0, rows, first_a, first_b, rank, dim=dim), lambda g: srv.adapter_grad(x, dout, g, 0, first_a, first_b, rank),
             lambda g: srv.expert_matmul(x, g, 0, rows // 4, dim=dim), lambda g: srv.expert_matmul(dout, g, 0, 64, dim=1024, transposed=False),
             lambda g: srv.expert_grad(dout, x, g))
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, n // 3, n // 2, n], dtype=torch.int32, device="cuda")
    good = [call((order, offsets)) for call in calls]
    for wrong in (-1, n, 1 << 30, -(1 << 31)):
        bad = order.clone()
        bad[n // 2] = wrong
        for call in calls:
            call((bad, offsets))
            with pytest.raises(P.PSError) as e:
                srv.status()
            assert e.value.code == P.PS_EKEY
    for wrong in ([0, -5, n, 2 * n], [n, n, n, n], [5, 3, 2, 1], [0, 1 << 30, -(1 << 31), 7]):
        for call in calls:
            call((order, torch.tensor(wrong, dtype=torch.int32, device="cuda")))
            srv.status()
    for call, was in zip(calls, good):                                  # and nothing of it stays
        for got, want in zip(*((r if isinstance(r, tuple) else (r,)) for r in (call((order, offsets)), was))):
            assert torch.equal(got, want)


def test_gradients_of_millions_of_rows():
    """Chunks of more rows than a workgroup holds the numbers of; sums of numbers of 0 and 1, which are exact in 32 bits (below 8 x 2^21), in whatever order."""
    import torch
    from paper_2002_00655_amd import ps as P
    n, rank, rows, dim = 2_300_000, 64, 8, 1024
    g = torch.Generator(device="cuda").manual_seed(5)
    values = torch.randint(0, 2, (rows + 4 * rank, dim), device="cuda", generator=g).float()
    srv = P.ParameterServer(values.shape[0], dim, 1)
    srv.push(torch.arange(values.shape[0], device="cuda"), values)
    x, dout = (torch.randint(0, 2, (n, c), device="cuda", generator=g, dtype=torch.int8).bfloat16() for c in (dim, rows))
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < 0.6, 1, 0)
    _, da, db = srv.adapter_grad(x, dout, srv.group_rows(ids, 2), 0, rows, rows + 2 * rank, rank, want_dx=False)
    for e in range(2):
        low = dout.double() @ values[rows + (2 + e) * rank:rows + (3 + e) * rank, :rows].double().t() * (ids == e)[:, None]
        want = sum(low[i:i + 100_000].t() @ x[i:i + 100_000].double() for i in range(0, n, 100_000))
        assert want.max() < 2 ** 24 and torch.equal(da[e].double(), want), e
    srv.status()


def test_gradients_against_differences():
    import torch
    case = (9, 3, 4, 20, 24, 24)
    n, adapters, rank, rows, dim, L = case
    srv, (first, first_a, first_b), w, a, b, ids = _setup(case)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), adapters, pad=-1)
    x, probe = _randn(6, n, dim), _randn(7, n, rows)
    dx, da, db = (t.double().cpu() for t in srv.adapter_grad(x.cuda(), probe.cuda(), groups, first, first_a, first_b, rank, scale=1.5))

    def value(x, a, b):
        return float((_forward(x, w, a, b, ids, 1.5)[0] * probe.double()).sum())
    rng, h = np.random.default_rng(0), 1e-3
    for _ in range(20):
        for which, grad in ((0, dx), (1, da), (2, db)):
            at = tuple(rng.integers(s) for s in grad.shape)
            values = []
            for sign in (1, -1):
                args = [x.double().clone(), a.clone(), b.clone()]
                args[which][at] += sign * h
                values.append(value(*args))
            assert abs((values[0] - values[1]) / (2 * h) - grad[at]) < 1e-4              # (linear in each: see the products with experts)


@pytest.mark.parametrize("caches", [False, True])
def test_statistics(caches):
    """A pull of W's keys and of both matrices of every adapter that is named, once each."""
    import torch
    from paper_2002_00655_amd import ps as P
    a, b = (P.ParameterServer(100, 16, 4) for _ in range(2))
    for s in (a, b):
        if caches:
            s.set_option(P.OPT_LOCATION_CACHES, 1)
        s.localize(torch.arange(10, 70, device="cuda"), 3)
    groups = a.group_rows(torch.tensor([5, -1, 2, 5], device="cuda"), 8, pad=-1)
    keys = torch.cat([torch.arange(4, 14)] + [f + e * 3 + torch.arange(3) for f in (20, 60) for e in (2, 5)]).cuda()
    x = torch.ones(4, 16, device="cuda")
    for worker in (0, 3):
        a.adapter_matmul(x, groups, 4, 10, 20, 60, 3, worker=worker)
        b.pull(keys, worker=worker)
        assert a.stats() == b.stats()
        a.adapter_grad(x, torch.ones(4, 10, device="cuda"), groups, 4, 20, 60, 3, worker=worker)
        b.pull(keys, worker=worker)
        assert a.stats() == b.stats()


def test_refusals_and_no_rows():
    import torch
    from paper_2002_00655_amd import ps as P
    srv, _ = _server(60, 16)
    groups = srv.group_rows(torch.zeros(5, dtype=torch.int64, device="cuda"), 4)
    x = torch.zeros(5, 16, device="cuda")

    def code(f):
        with pytest.raises(P.PSError) as e:
            f()
        return e.value.code
    assert code(lambda: srv.adapter_matmul(x, groups, 50, 16, 0, 20, 4)) == P.PS_EINVAL        # W past the last key
    assert code(lambda: srv.adapter_matmul(x, groups, 0, 16, 45, 20, 4)) == P.PS_EINVAL        # A
    assert code(lambda: srv.adapter_matmul(x, groups, 0, 16, 20, 45, 4)) == P.PS_EINVAL        # B
    assert code(lambda: srv.adapter_matmul(x, groups, 0, 17, 20, 40, 4)) == P.PS_EINVAL        # more rows than a key has values
    assert code(lambda: srv.adapter_matmul(x, groups, 0, 16, 20, 40, 0)) == P.PS_EINVAL
    assert code(lambda: srv.adapter_matmul(x, groups, 0, 16, 20, 40, 4, worker=2)) == P.PS_EWORKER
    for wrong in (x[:4], x[:, :8], x.t()):
        with pytest.raises(ValueError):
            srv.adapter_matmul(wrong, groups, 0, 16, 20, 40, 4)
    with pytest.raises(TypeError):
        srv.adapter_grad(x, x.half(), groups, 0, 20, 40, 4)
    none = srv.group_rows(torch.zeros(0, dtype=torch.int64, device="cuda"), 4)
    assert srv.adapter_matmul(x[:0], none, 0, 16, 20, 40, 4).shape == (0, 16)
    dx, da, db = srv.adapter_grad(x[:0], x[:0], none, 0, 20, 40, 4)
    assert dx.shape == (0, 16) and (da == 0).all() and (db == 0).all()
    order = torch.arange(5, dtype=torch.int32, device="cuda")
    order[3] = 9
    srv.adapter_matmul(x, (order, groups[1]), 0, 16, 20, 40, 4)
    with pytest.raises(P.PSError):
        srv.status()
    for wrong in ([0, -5, 7, 2, 5], [5, 4, 3, 2, 1], [0, 1 << 30, -(1 << 31), 7, 7]):
        offsets = torch.tensor(wrong, dtype=torch.int32, device="cuda")
        srv.adapter_matmul(x, (groups[0], offsets), 0, 16, 20, 40, 4)
        srv.adapter_grad(x, x, (groups[0], offsets), 0, 20, 40, 4)
        srv.status()


@pytest.mark.parametrize("n", [48, 2500])
def test_captured_and_replayed(n):
    import torch
    case = (n, 6, 16, 256, 128, 256)
    srv, (first, first_a, first_b), *_ = _setup(case)
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    x, dout = torch.zeros(n, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 256, dtype=torch.bfloat16, device="cuda")

    def step():
        groups = srv.group_rows(ids, 6, pad=-1)
        return (srv.adapter_matmul(x, groups, first, 256, first_a, first_b, 16, dim=128), *srv.adapter_grad(x, dout, groups, first, first_a, first_b, 16))
    step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = step()
    torch.cuda.current_stream().wait_stream(stream)
    g = torch.Generator(device="cuda").manual_seed(5)
    for i in range(4):
        ids.copy_(torch.randint(-1, 2 + i, ids.shape, device="cuda", generator=g))
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        dout.copy_(torch.randn(dout.shape, device="cuda", generator=g))
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
    srv.status()


def test_a_step_of_adapters():
    """Adapters trained in the server: forward, gradients, and their rows stepped by AdaGrad with the keys as tokens - against the same in 64 bits."""
    import torch
    from paper_2002_00655_amd import ps as P
    adapters, rank, rows, dim, n, L = 4, 6, 40, 32, 200, 80
    first, first_a, first_b = 0, rows, rows + adapters * rank
    keys = first_b + adapters * rank
    values = torch.randn(keys, L, generator=torch.Generator().manual_seed(3)) * 0.1
    values[first_a:first_b, dim:2 * dim] = 0
    values[first_b:, rows:2 * rows] = 0
    srv = P.ParameterServer(keys, L, 1)
    srv.push(torch.arange(keys, device="cuda"), values.cuda())
    ids = torch.from_numpy(np.random.default_rng(1).integers(-1, adapters, size=n))
    x, target = _randn(1, n, dim), _randn(2, n, rows)
    groups = srv.group_rows(ids.cuda(), adapters, pad=-1)
    y = srv.adapter_matmul(x.cuda(), groups, first, rows, first_a, first_b, rank, scale=2.0, dim=dim)
    dx, da, db = srv.adapter_grad(x.cuda(), 2 * (y - target.cuda()), groups, first, first_a, first_b, rank, scale=2.0)
    a_keys, b_keys = (torch.arange(adapters * rank, device="cuda") for _ in range(2))
    srv.emb_adagrad_step(a_keys, da.view(-1, dim), 0.1, 1e-8, first_key=first_a, num_tokens=adapters * rank)
    srv.emb_adagrad_step(b_keys, db.view(-1, rows), 0.1, 1e-8, first_key=first_b, num_tokens=adapters * rank)
    got = srv.pull(torch.arange(keys, device="cuda")).double().cpu()

    v = values.double()
    w, a, b = v[:rows, :dim], v[first_a:first_b, :dim].reshape(adapters, rank, dim).clone().requires_grad_(), v[first_b:, :rows].reshape(adapters, rank, rows).clone().requires_grad_()
    out = torch.stack([w @ x.double()[p] + (2.0 * (a[e] @ x.double()[p]) @ b[e] if e >= 0 else 0) for p, e in enumerate(ids.tolist())])
    ((out - target.double()) ** 2).sum().backward()
    # a first step of AdaGrad is lr g / sqrt(g^2 + eps): lr times its sign, where g is far from 0
    for grad, start, cols in ((a.grad.reshape(-1, dim), first_a, dim), (b.grad.reshape(-1, rows), first_b, rows)):
        moved = got[start:start + adapters * rank, :cols] - v[start:start + adapters * rank, :cols]
        large = grad.abs() > 1e-2
        assert large.float().mean() > 0.9
        assert ((moved + 0.1 * grad / (grad ** 2 + 1e-8).sqrt()).abs()[large] < 1e-4).all()
    srv.status()
