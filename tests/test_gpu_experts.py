"""Rows by group, products with experts and their gradients against the formulas in 64 bits: types, sizes on both sides of every rule, odd sides, strides and
alignments, shared rows and sums of pairs, groups without rows, rows of no group, numbers that are none where nothing is read; refusals, graphs, streams.

Tolerances, element by element, relative to S, the sum of the absolute values of the terms: a sum of K terms on the matrix cores is off by at most K + 8 units of
2^-23 (its additions need not round to the nearest); where products are of 16 bits, a number of the server is off by half a step of that type (2^-8, 2^-11), or,
for fp16, by 2^-25 where it is smaller than the smallest normal number; the result by half a step of its own type, or 2^-25 (fp16)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _type(name):
    import torch
    return getattr(torch, name)


def _server(K, L, seed=0, scale=0.05, W=1):
    import torch
    from paper_2002_00655_amd import ps as P
    values = torch.randn(K, L, generator=torch.Generator().manual_seed(seed)) * scale
    srv = P.ParameterServer(K, L, W)
    srv.push(torch.arange(K, device="cuda"), values.cuda())
    return srv, values


def _randn(seed, *shape, kind="float32", scale=1.0):
    import torch
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(_type(kind))


def _order(ids, groups, pad):
    key = np.where(ids == pad, groups, ids) if pad is not None else ids
    return np.argsort(key, kind="stable"), np.array([(key < e).sum() for e in range(groups + 1)])


def _close(got, want, mag, rel, kind, extra=0.0):
    """|got - want| <= rel mag + half a step of the result's type"""
    got = got.double().cpu()
    tol = rel * mag + HALF[kind] * want.abs() * (1 + rel) + (2.0 ** -25 if kind == "float16" else 1e-37) + extra
    bad = (got - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / tol).max()))


def _product(x, w, ids, per, transposed):
    """The rows' products and the sums of their terms' absolute values, in 64 bits: rows of no group zero.  w: [experts, rows, dim]"""
    import torch
    n, cols = ids.size, w.shape[2] if transposed else w.shape[1]
    x, w = x.double(), w.double()
    out, mag = torch.zeros(n, cols, dtype=torch.float64), torch.zeros(n, cols, dtype=torch.float64)
    for e in range(w.shape[0]):
        q = torch.from_numpy(np.nonzero(ids == e)[0])
        m = w[e] if transposed else w[e].t()
        out[q], mag[q] = x[q // per] @ m, x[q // per].abs() @ m.abs()
    return out, mag


def _terms_off(kind, precise, K):
    return (K + 8) * 2.0 ** -23 + (0.0 if precise else HALF[kind] * (1 + 2.0 ** -10))


# ---- group_rows -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1000, 1023, 4095, 4096, 4097, 20001, 131073])
@pytest.mark.parametrize("groups", [1, 2, 7, 64, 511, 2046, 2047, 5000])
def test_group_rows(n, groups):
    import torch
    print(f"case n={n} groups={groups}", flush=True)
    srv, _ = _server(1, 1)
    rng = np.random.default_rng(n * 7 + groups)
    for wide in (False, True):
        for pad in (None, -1, 0, 10 ** 6):
            ids = rng.integers(0, groups, size=n)
            if groups > 4 and n:
                ids[rng.random(n) < 0.5] = groups // 2                   # one group of many rows, others of few or none
            if pad is not None:
                ids[rng.random(n) < 0.2] = pad
            order, offsets = srv.group_rows(torch.from_numpy(ids.astype(np.int64 if wide else np.int32)).cuda(), groups, pad=pad)
            want, starts = _order(ids, groups, pad)
            assert order.dtype == offsets.dtype == torch.int32
            np.testing.assert_array_equal(offsets.cpu().numpy(), starts)
            np.testing.assert_array_equal(order.cpu().numpy(), want)
    srv.status()


def test_group_rows_of_millions():
    """More rows than workgroups count by themselves: by a sort."""
    import torch
    srv, _ = _server(1, 1)
    n, groups = 128 * 16384 + 5, 300
    ids = torch.randint(-1, groups, (n,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    order, offsets = srv.group_rows(ids, groups, pad=-1)
    key = torch.where(ids < 0, torch.full_like(ids, groups), ids)
    assert torch.equal(order.long(), torch.sort(key, stable=True).indices)
    assert torch.equal(offsets.long(), torch.searchsorted(torch.sort(key).values, torch.arange(groups + 1, device="cuda", dtype=torch.int32)))


@pytest.mark.parametrize("n,groups", [(3, 4), (4096, 16), (5000, 16), (70, 3000), (5000, 3000)])
@pytest.mark.parametrize("bad", [-2, -(1 << 40), 1 << 40, None])
def test_group_rows_refuses_ids_out_of_range(n, groups, bad):
    """Nothing is written, and nothing by later calls, until the error has been asked for."""
    import torch
    from paper_2002_00655_amd import ps as P
    srv, _ = _server(1, 1)
    ids = torch.arange(n, device="cuda") % groups
    ids[n // 2] = groups if bad is None else bad
    order, offsets = torch.full((n,), 77, device="cuda", dtype=torch.int32), torch.full((groups + 1,), 77, device="cuda", dtype=torch.int32)

    def call(ids):
        return P._lib.group_rows(srv._h, groups, ids.data_ptr(), 1, n, -1, order.data_ptr(), offsets.data_ptr(), P._stream())
    assert call(ids) == 0
    good = torch.arange(n, device="cuda") % groups
    assert call(good) == 0
    assert (order == 77).all() and (offsets == 77).all()
    with pytest.raises(P.PSError) as e:
        srv.status()
    assert e.value.code == P.PS_EKEY
    assert call(good) == 0
    srv.status()
    np.testing.assert_array_equal(order.cpu().numpy(), _order(good.cpu().numpy(), groups, None)[0])


# ---- expert_matmul --------------------------------------------------------------------------------------------------
# sizes on both sides of what decides between the kernels: few rows, columns of at most 32, tiles of 64, of 128, laid matrices
CASES = [
    # n, experts, rows, dim, L, first
    (1, 3, 1, 1, 1, 0),
    (1, 8, 64, 64, 64, 5),
    (2, 1, 16, 100, 128, 0),
    (17, 5, 33, 127, 127, 3),
    (130, 4, 31, 65, 130, 7),
    (700, 3, 32, 96, 200, 0),
    (333, 7, 129, 51, 53, 2),
    (1500, 70, 65, 33, 66, 1),
    (2000, 2, 260, 256, 512, 0),
    (2500, 5, 200, 1024, 1024, 11),
    (4100, 1, 1030, 72, 73, 0),
    (9000, 2, 515, 264, 264, 0),
    (16400, 3, 2050, 40, 41, 0),                     # (laid)
    (33000, 2, 48, 1000, 1000, 0),                   # (laid, transposed)
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
def test_expert_matmul(case, kind, transposed):
    import torch
    n, experts, rows, dim, L, first = case
    print("case", case, kind, transposed, flush=True)
    srv, values = _server(first + experts * rows + 3, L, seed=n)
    w = values[first:first + experts * rows, :dim].reshape(experts, rows, dim)
    K, N = (rows, dim) if transposed else (dim, rows)
    rng = np.random.default_rng(n + rows)
    for pad, skew in ((None, False), (-1, True)):
        ids = rng.integers(0, experts, size=n)
        if skew:
            ids[rng.random(n) < 0.6] = experts - 1
            ids[rng.random(n) < 0.2] = -1
        groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts, pad=pad)
        x = _randn(n + 1, n, K, kind=kind)
        want, mag = _product(x, w, ids, 1, transposed)
        for out_kind in (kind, "float32", "bfloat16" if kind == "float32" else kind):
            out = srv.expert_matmul(x.cuda(), groups, first, rows, dim=dim, transposed=transposed, dtype=_type(out_kind))
            precise = "float32" in (kind, out_kind)
            small = 2.0 ** -25 * x.double().abs().sum(1).max().item() if kind == "float16" and not precise else 0.0
            _close(out, want, mag, _terms_off(kind, precise, K), out_kind, small)
            assert (out[torch.from_numpy(ids).cuda() == -1] == 0).all()
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,rows,dim", [(40, 48, 72), (900, 130, 200), (5200, 512, 520), (16500, 2056, 40)])
def test_expert_matmul_strides_and_numbers_that_are_none(kind, n, rows, dim):
    """Rows of x with gaps and at odd places, rows of the result with gaps; no number beside what belongs to a row, in the server or in x, has a part in it, and
    what lies between the rows of the result stays."""
    import torch
    experts, L = 3, 2 * dim + 1 if 2 * dim < 1024 else dim + 8
    print("case", kind, n, rows, dim, flush=True)
    srv, values = _server(experts * rows + 2, L, seed=3)
    spoil = torch.zeros_like(values)
    spoil[:, dim:] = float("nan")
    spoil[-2:] = float("inf")
    srv.push(torch.arange(values.shape[0], device="cuda"), spoil.cuda())
    w = values[:experts * rows, :dim].reshape(experts, rows, dim)
    ids = np.random.default_rng(1).integers(0, experts, size=n)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts)
    for transposed in (False, True):
        K, N = (rows, dim) if transposed else (dim, rows)
        x = _randn(5, n, K, kind=kind)
        want, mag = _product(x, w, ids, 1, transposed)
        small = 2.0 ** -25 * x.double().abs().sum(1).max().item() if kind == "float16" else 0.0
        for before, gap in ((0, 0), (1, 0), (0, 3), (8, 8), (3, 5)):
            frame = torch.full((n + 2, before + K + gap), float("nan"), dtype=_type(kind), device="cuda")
            view = frame[1:-1, before:before + K]
            view.copy_(x)
            to = torch.full((n + 2, before + N + gap), 7.0, dtype=_type(kind), device="cuda")
            out = to[1:-1, before:before + N]
            assert srv.expert_matmul(view, groups, 0, rows, dim=dim, transposed=transposed, out=out) is out
            _close(out, want, mag, _terms_off(kind, kind == "float32", K), kind, small)
            out.fill_(7.0)
            assert (to == 7.0).all()
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [33, 600, 5000])
def test_a_row_that_is_no_number_spoils_no_other(kind, n):
    """Infinities and NaN of a row of x, of one expert's matrix, of rows of no group."""
    import torch
    experts, rows, dim = 4, 136, 264
    srv, values = _server(experts * rows, 264, seed=4)
    bad = torch.zeros_like(values)
    bad[2 * rows + 5, 7] = float("nan")
    srv.push(torch.arange(values.shape[0], device="cuda"), bad.cuda())
    ids = np.random.default_rng(2).integers(-1, experts, size=n)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts, pad=-1)
    for transposed in (False, True):
        x = _randn(6, n, rows if transposed else dim, kind=kind)
        clean = srv.expert_matmul(x.cuda(), groups, 0, rows, transposed=transposed)
        x[0, 3], x[n // 2, 0], x[n - 1, -1] = float("inf"), float("nan"), -float("inf")
        x[torch.from_numpy(np.nonzero(ids == -1)[0][:3])] = float("nan")
        out = srv.expert_matmul(x.cuda(), groups, 0, rows, transposed=transposed)
        touched = torch.zeros(n, dtype=torch.bool)
        touched[[0, n // 2, n - 1]] = True
        ids_t = torch.from_numpy(ids)
        keep = ~touched | (ids_t == -1)
        assert torch.equal(torch.nan_to_num(out[keep.cuda()].float(), nan=123.0), torch.nan_to_num(clean[keep.cuda()].float(), nan=123.0))
        assert (out[(ids_t == -1).cuda()] == 0).all()
        good = (ids_t != 2) & keep
        assert torch.isfinite(out[good.cuda()].float()).all()
        spoiled = out[((ids_t == 2)).cuda()].float()
        assert spoiled.numel() == 0 or (torch.isnan(spoiled).any(1).all())
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("tokens,k", [(1, 2), (37, 3), (500, 4), (4100, 2)])
def test_pairs(kind, tokens, k):
    """Rows of x that stand for several, and sums of neighbouring rows: a token's choices, there and back."""
    import torch
    experts, rows, dim = 6, 144, 104
    srv, values = _server(experts * rows, 2 * dim, seed=7)
    w = values[:, :dim].reshape(experts, rows, dim)
    rng = np.random.default_rng(tokens)
    ids = np.stack([rng.permutation(experts)[:k] for _ in range(tokens)]).reshape(-1)
    ids[rng.random(ids.size) < 0.2] = -1
    groups = srv.group_rows(torch.from_numpy(ids.reshape(tokens, k)).cuda(), experts, pad=-1)
    x = _randn(8, tokens, dim, kind=kind)
    want, mag = _product(x, w, ids, k, False)
    small = 2.0 ** -25 * x.double().abs().sum(1).max().item() if kind == "float16" else 0.0
    _close(srv.expert_matmul(x.cuda(), groups, 0, rows, dim=dim), want, mag, _terms_off(kind, kind == "float32", dim), kind, small)
    h = _randn(9, tokens * k, rows, kind=kind)
    want, mag = _product(h, w, ids, 1, True)
    want, mag = want.view(tokens, k, dim).sum(1), mag.view(tokens, k, dim).sum(1)
    out = srv.expert_matmul(h.cuda(), groups, 0, rows, dim=dim, transposed=True, sum_pairs=k)
    assert out.shape == (tokens, dim)
    _close(out, want, mag, _terms_off(kind, kind == "float32", rows + k), kind, k * 2.0 ** -25 * h.double().abs().sum(1).max().item() if kind == "float16" else 0.0)
    again = srv.expert_matmul(h.cuda(), groups, 0, rows, dim=dim, transposed=True, sum_pairs=k, out=torch.empty_like(out))
    assert torch.equal(again, out)                                      # the order of additions depends on the arguments only
    # one row for all: not copied
    one = x[:1].cuda().expand(tokens, dim)
    want, mag = _product(x[:1].expand(tokens, dim), w, ids, k, False)
    _close(srv.expert_matmul(one, groups, 0, rows, dim=dim), want, mag, _terms_off(kind, kind == "float32", dim), kind, small)


@pytest.mark.parametrize("dim", [7, 8])
def test_beyond_32_bits(dim):
    """Matrices at the end of a server of more than 2^31 numbers, rows and results of as many; numbers of 0 and 1, whose sums are exact."""
    import torch
    from paper_2002_00655_amd import ps as P
    n, rows, experts, L = 2_200_002, 1024, 2, 1024
    first = 2_200_000
    srv = P.ParameterServer(first + experts * rows, L, 1)
    g = torch.Generator(device="cuda").manual_seed(dim)
    w = torch.randint(0, 2, (experts * rows, L), device="cuda", generator=g).float()
    srv.push(torch.arange(first, first + experts * rows, device="cuda"), w)
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < 0.6, 1, 0)
    ids[::19] = -1
    groups = srv.group_rows(ids, experts, pad=-1)
    x = torch.zeros(n, 1024, dtype=torch.bfloat16, device="cuda")[:, :dim]
    x.copy_(torch.randint(0, 2, (n, dim), device="cuda", generator=g))
    out = srv.expert_matmul(x, groups, first, rows, dim=dim)
    back = srv.expert_matmul(out, groups, first, rows, dim=dim, transposed=True, sum_pairs=2, dtype=torch.float32)
    m = w.view(experts, rows, L)[:, :, :dim]
    for i in range(0, n, 200_000):
        j = min(n, i + 200_000)
        one = torch.stack([(ids[i:j] == e).float() for e in range(experts)])
        want = sum((x[i:j].float() * one[e][:, None]) @ m[e].t() for e in range(experts))
        assert torch.equal(out[i:j].float(), want), i
        want = sum((want * one[e][:, None]) @ m[e] for e in range(experts))
        assert torch.equal(back[i // 2:j // 2], want.view(-1, 2, dim).sum(1)), i
    srv.status()


# ---- expert_grad ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,experts,rows,dim", [(0, 3, 5, 7), (1, 2, 1, 1), (5, 9, 16, 24), (200, 3, 64, 65), (333, 5, 100, 127), (700, 4, 72, 136), (3000, 2, 136, 264),
                                                (9000, 3, 40, 300), (6001, 2, 129, 130), (5000, 200, 8, 8)])
def test_expert_grad(kind, n, experts, rows, dim):
    import torch
    print("case", kind, n, experts, rows, dim, flush=True)
    srv, _ = _server(1, 1)
    rng = np.random.default_rng(n)
    for per_left, per_right in ((1, 1), (1, 2), (2, 1)):
        m = n // 2 * 2 if 2 in (per_left, per_right) else n
        ids = rng.integers(0, experts, size=m)
        ids[rng.random(m) < 0.5] = 0
        ids[rng.random(m) < 0.1] = -1
        if experts > 2:
            ids[ids == 1] = 2                                           # a group without rows
        groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts, pad=-1)
        left, right = _randn(n + 1, m // per_left, rows, kind=kind), _randn(n + 2, m // per_right, dim, kind=kind)
        want, mag = torch.zeros(experts, rows, dim, dtype=torch.float64), torch.zeros(experts, rows, dim, dtype=torch.float64)
        for e in range(experts):
            q = torch.from_numpy(np.nonzero(ids == e)[0])
            a, b = left.double()[q // per_left], right.double()[q // per_right]
            want[e], mag[e] = a.t() @ b, a.abs().t() @ b.abs()
        for out_kind in ("float32", kind):
            out = srv.expert_grad(left.cuda(), right.cuda(), groups, dtype=_type(out_kind))
            assert out.shape == want.shape
            _close(out, want, mag, (np.bincount(ids[ids >= 0], minlength=1).max() + 40) * 2.0 ** -23 if m else 0.0, out_kind)
        assert torch.equal(srv.expert_grad(left.cuda(), right.cuda(), groups, dtype=_type(kind)), out)
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,side", [(9000, 4096), (20001, 2056)])
def test_expert_grad_of_large_matrices(kind, n, side):
    """Chunks of more rows than a workgroup holds the numbers of; sums of numbers of -1, 0 and 1, which are exact in 32 bits, in whatever order."""
    import torch
    print("case", kind, n, side, flush=True)
    srv, _ = _server(1, 1)
    g = torch.Generator(device="cuda").manual_seed(n)
    left, right = (torch.randint(-1, 2, (n, side), device="cuda", generator=g).to(_type(kind)) for _ in range(2))
    ids = torch.where(torch.rand(n, device="cuda", generator=g) < 0.9, 2, 0)
    ids[::17] = -1
    out = srv.expert_grad(left, right, srv.group_rows(ids, 3, pad=-1))
    for e in range(3):
        q = (ids == e).nonzero()[:, 0]
        assert torch.equal(out[e].double(), left[q].double().t() @ right[q].double()), e
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
def test_expert_grad_strides_and_numbers_that_are_none(kind):
    import torch
    srv, _ = _server(1, 1)
    n, experts, rows, dim = 700, 3, 104, 72
    ids = np.random.default_rng(3).integers(-1, experts, size=n)
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts, pad=-1)
    left, right = _randn(1, n, rows, kind=kind), _randn(2, n, dim, kind=kind)
    left[torch.from_numpy(np.nonzero(ids == -1)[0])] = float("nan")     # rows of no group
    want = torch.stack([left.double()[torch.from_numpy(ids == e)].t() @ right.double()[torch.from_numpy(ids == e)] for e in range(experts)])
    mag = torch.stack([left.double()[torch.from_numpy(ids == e)].abs().t() @ right.double()[torch.from_numpy(ids == e)].abs() for e in range(experts)])
    for before, gap in ((0, 0), (1, 0), (8, 8), (0, 5), (16, 40)):
        views = []
        for t in (left, right):
            frame = torch.full((n + 2, before + t.shape[1] + gap), float("nan"), dtype=t.dtype, device="cuda")
            frame[1:-1, before:before + t.shape[1]].copy_(t)
            views.append(frame[1:-1, before:before + t.shape[1]])
        _close(srv.expert_grad(*views, groups), want, mag, (n + 40) * 2.0 ** -23, "float32")
    # an infinity of one group is in its matrix alone
    left[torch.from_numpy(np.nonzero(ids == 1)[0][:1]), 5] = float("inf")
    out = srv.expert_grad(left.cuda(), right.cuda(), groups)
    assert torch.isfinite(out[[0, 2]]).all() and not torch.isfinite(out[1, 5]).any() and torch.isfinite(out[1, :5]).all()


def test_gradients_against_differences():
    """dx and dW of a scalar of the products, against its differences in 64 bits of the formula."""
    import torch
    experts, rows, dim, tokens, k = 3, 24, 40, 7, 2
    srv, values = _server(experts * rows, dim, seed=1, scale=0.2)
    w = values.reshape(experts, rows, dim).double()
    ids = np.array([[0, 1], [1, 2], [2, 0], [0, 2], [1, 0], [-1, 1], [2, -1]])
    groups = srv.group_rows(torch.from_numpy(ids).cuda(), experts, pad=-1)
    x, probe = _randn(2, tokens, dim), _randn(3, tokens * k, rows)
    dx = srv.expert_matmul(probe.cuda(), groups, 0, rows, transposed=True, sum_pairs=k).double().cpu()
    dw = srv.expert_grad(probe.cuda(), x.cuda(), groups).double().cpu()

    def value(x, w):
        return float(sum((w[e] @ x[p // k]) @ probe.double()[p] for p, e in enumerate(ids.reshape(-1)) if e >= 0))
    rng, h = np.random.default_rng(0), 1e-3
    for _ in range(20):
        t, c = rng.integers(tokens), rng.integers(dim)
        up, down = x.double().clone(), x.double().clone()
        up[t, c] += h
        down[t, c] -= h
        assert abs((value(up, w) - value(down, w)) / (2 * h) - dx[t, c]) < 1e-4       # (the value is linear: what is left is 2^-53 of it over 2 h, and dx in 32 bits)
        e, r = rng.integers(experts), rng.integers(rows)
        up, down = w.clone(), w.clone()
        up[e, r, c] += h
        down[e, r, c] -= h
        assert abs((value(x.double(), up) - value(x.double(), down)) / (2 * h) - dw[e, r, c]) < 1e-4


# ---- statistics, orders that are none, refusals, graphs, streams -----------------------------------------------------
@pytest.mark.parametrize("caches", [False, True])
def test_statistics(caches):
    """A product is a pull of the keys of the experts that have rows, once each."""
    import torch
    from paper_2002_00655_amd import ps as P
    experts, rows, dim, first = 5, 12, 8, 3
    a, b = (P.ParameterServer(100, 8, 4) for _ in range(2))
    for s in (a, b):
        if caches:
            s.set_option(P.OPT_LOCATION_CACHES, 1)
        s.localize(torch.arange(20, 50, device="cuda"), 2)
    ids = torch.tensor([0, 4, 4, 1, -1, 0], device="cuda")
    groups = a.group_rows(ids, experts, pad=-1)
    keys = torch.cat([first + e * rows + torch.arange(rows) for e in (0, 1, 4)]).cuda()
    x = torch.ones(6, dim, device="cuda")
    for worker in (1, 2, 3):
        a.expert_matmul(x, groups, first, rows, dim=dim, worker=worker)
        b.pull(keys, worker=worker)
        assert a.stats() == b.stats()
    a.expert_matmul(x, groups, first, rows, dim=dim)
    a.expert_grad(torch.ones(6, rows, device="cuda"), x, groups)
    assert a.stats() == b.stats()


def test_orders_that_are_none_do_no_harm():
    """Numbers out of range are found where they are read; rows that stand nowhere in the order stay as they are."""
    import torch
    from paper_2002_00655_amd import ps as P
    experts, rows, dim = 3, 40, 48
    for n in (10, 700):
        srv, _ = _server(experts * rows, dim)
        x = torch.randn(n, dim, device="cuda")
        offsets = torch.tensor([0, n // 3, n // 2, n], dtype=torch.int32, device="cuda")
        for wrong in (-1, n, 1 << 30, -(1 << 31)):
            order = torch.arange(n, dtype=torch.int32, device="cuda")
            order[n // 2] = wrong
            for call in (lambda: srv.expert_matmul(x, (order, offsets), 0, rows), lambda: srv.expert_grad(x, x, (order, offsets))):
                call()
                with pytest.raises(P.PSError) as e:
                    srv.status()
                assert e.value.code == P.PS_EKEY
        order = torch.arange(n, dtype=torch.int32, device="cuda")
        good = srv.expert_matmul(x, (order, offsets), 0, rows)
        for wrong in ([0, -5, n, 2 * n], [n, n, n, n], [5, 3, 2, 1], [0, 1 << 30, -(1 << 31), 7]):
            wrong = torch.tensor(wrong, dtype=torch.int32, device="cuda")
            srv.expert_matmul(x, (order, wrong), 0, rows)
            srv.expert_grad(x, x, (order, wrong))
            srv.status()
        # a row that stands nowhere
        order[4] = 5
        out = torch.full((n, rows), 7.0, device="cuda")
        srv.expert_matmul(x, (order, offsets), 0, rows, out=out)
        assert (out[4] == 7.0).all() and torch.equal(out[:4], good[:4]) and torch.equal(out[6:], good[6:])
        srv.status()


def test_refusals():
    import torch
    from paper_2002_00655_amd import ps as P
    srv, _ = _server(40, 16)
    ids = torch.zeros(6, dtype=torch.int64, device="cuda")
    groups = srv.group_rows(ids, 2)
    x = torch.zeros(6, 16, device="cuda")

    def code(f):
        with pytest.raises(P.PSError) as e:
            f()
        return e.value.code
    assert code(lambda: srv.group_rows(ids, 0)) == P.PS_EINVAL
    assert code(lambda: srv.group_rows(ids, 65537)) == P.PS_ELIMIT
    for wrong in (ids.cpu(), ids.float(), ids[::2]):
        with pytest.raises(TypeError):
            srv.group_rows(wrong, 2)
    assert code(lambda: srv.expert_matmul(x, groups, 1, 20)) == P.PS_EINVAL            # past the last key
    assert code(lambda: srv.expert_matmul(x, groups, -1, 20)) == P.PS_EINVAL
    assert code(lambda: srv.expert_matmul(torch.zeros(6, 17, device="cuda"), groups, 0, 20, dim=17)) == P.PS_EINVAL
    assert code(lambda: srv.expert_matmul(x, groups, 0, 20, worker=1)) == P.PS_EWORKER
    with pytest.raises(ValueError):
        srv.expert_matmul(x[:, :8], groups, 0, 20)
    with pytest.raises(ValueError):
        srv.expert_matmul(x[:4], groups, 0, 20)
    with pytest.raises(ValueError):
        srv.expert_matmul(x.t().contiguous().t(), groups, 0, 20)                       # columns
    with pytest.raises(ValueError):
        srv.expert_matmul(x, groups, 0, 20, sum_pairs=4)
    with pytest.raises(ValueError):
        srv.expert_matmul(x, groups, 0, 20, out=torch.zeros(6, 19, device="cuda"))
    with pytest.raises(TypeError):
        srv.expert_matmul(x.double(), groups, 0, 20)
    with pytest.raises(TypeError):
        srv.expert_matmul(x, groups, 0, 20, dtype=torch.float64)
    with pytest.raises(TypeError):
        srv.expert_matmul(x, (groups[0].long(), groups[1]), 0, 20)
    with pytest.raises(TypeError):
        srv.expert_grad(x, x.half(), groups)
    with pytest.raises(ValueError):
        srv.expert_grad(x[:5], x, groups)
    assert P._lib.expert_matmul(srv._h, -1, 0, 2, 20, 16, 0, *[g.data_ptr() for g in groups], 6, x.data_ptr(), 0, 1 << 31, 1, x.data_ptr(), 0, 20, 1, P._stream()) == P.PS_ELIMIT
    # no rows at all
    none = srv.group_rows(ids[:0], 2)
    assert srv.expert_matmul(x[:0], none, 0, 20).shape == (0, 20)
    assert (srv.expert_grad(x[:0], x[:0], none) == 0).all()
    srv.status()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_captured_and_replayed(kind):
    """The calls of a step in a graph: replayed with other rows and other groups, with work of the program between the replays, each against the calls themselves."""
    import torch
    experts, rows, dim, tokens, k = 4, 136, 128, 1500, 2
    srv, values = _server(experts * rows, 2 * dim, seed=2)
    ids = torch.zeros(tokens, k, dtype=torch.int32, device="cuda")
    x, dout = torch.zeros(tokens, dim, dtype=_type(kind), device="cuda"), torch.zeros(tokens * k, rows, dtype=_type(kind), device="cuda")

    def step():
        groups = srv.group_rows(ids, experts, pad=-1)
        return (srv.expert_matmul(x, groups, 0, rows, dim=dim), srv.expert_matmul(dout, groups, 0, rows, dim=dim, transposed=True, sum_pairs=k), srv.expert_grad(dout, x, groups))
    step()                                                              # (scratch grows)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = step()
    torch.cuda.current_stream().wait_stream(stream)
    g = torch.Generator(device="cuda").manual_seed(5)
    for i in range(4):
        ids.copy_(torch.randint(-1, 1 + i, ids.shape, device="cuda", generator=g))
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        dout.copy_(torch.randn(dout.shape, device="cuda", generator=g))
        graph.replay()
        got = [t.clone() for t in held]
        srv.push(torch.arange(experts * rows, device="cuda"), torch.zeros(experts * rows, 2 * dim, device="cuda"))      # the handle's scratch is used in between
        torch.cuda.synchronize()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
    srv.status()


def test_on_another_stream():
    import torch
    experts, rows, dim, n = 3, 72, 136, 900
    srv, values = _server(experts * rows, dim)
    ids = torch.randint(0, experts, (n,), device="cuda")
    x = torch.randn(n, dim, device="cuda").bfloat16()
    want = srv.expert_matmul(x, srv.group_rows(ids, experts), 0, rows)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(2_000_000)
        late = x.clone().mul_(2)
        out = srv.expert_matmul(late, srv.group_rows(ids, experts), 0, rows)
    stream.synchronize()
    assert torch.equal(out, (want.float() * 2).bfloat16())


def test_a_step_of_a_mixture():
    """The calls as a model's step uses them: rows chosen, up and down again, the gradients, and both matrices stepped in the server by their orthogonalised
    momentum - against the same in 64 bits, but for the step, whose own tests it has: here that the weights move against the gradient."""
    import torch
    experts, hidden, dim, tokens, k = 4, 96, 64, 300, 2
    keys = experts * hidden
    srv, values = _server(2 * keys, 2 * dim, seed=9, scale=0.1)
    values[:, dim:] = 0
    srv.push(torch.arange(2 * keys, device="cuda"), (values.cuda() - srv.pull(torch.arange(2 * keys, device="cuda"))))
    up, down = (values[i * keys:(i + 1) * keys, :dim].reshape(experts, hidden, dim).double().requires_grad_() for i in (0, 1))
    rng = np.random.default_rng(4)
    ids = torch.from_numpy(np.stack([rng.permutation(experts)[:k] for _ in range(tokens)]))
    gates, x, target = torch.rand(tokens * k, 1), _randn(1, tokens, dim), _randn(2, tokens, dim)

    xr = x.double().requires_grad_()
    h = torch.stack([torch.relu(up[e] @ xr[p // k]) * gates.double()[p] for p, e in enumerate(ids.reshape(-1).tolist())])
    y = torch.stack([down[e].t() @ h[p] for p, e in enumerate(ids.reshape(-1).tolist())]).view(tokens, k, dim).sum(1)
    ((y - target.double()) ** 2).sum().backward()

    groups = srv.group_rows(ids.cuda(), experts)
    xc, gc = x.cuda(), gates.cuda()
    a = srv.expert_matmul(xc, groups, 0, hidden, dim=dim)
    hc = torch.relu(a) * gc
    yc = srv.expert_matmul(hc, groups, keys, hidden, dim=dim, transposed=True, sum_pairs=k)
    dy = 2 * (yc - target.cuda())
    d_down = srv.expert_grad(hc, dy, groups)
    dh = srv.expert_matmul(dy, groups, keys, hidden, dim=dim) * gc * (a > 0)
    d_up = srv.expert_grad(dh, xc, groups)
    dx = srv.expert_matmul(dh, groups, 0, hidden, dim=dim, transposed=True, sum_pairs=k)
    # (a gradient goes through four sums of up to `terms` numbers of 32 bits one behind another, and sums of the errors of what goes into it)
    terms = 4 * (dim + hidden + k + tokens)
    for got, want in ((yc, y.detach()), (d_down, down.grad), (d_up, up.grad), (dx, xr.grad)):
        assert (got.double().cpu() - want).norm() <= terms * 2.0 ** -23 * want.norm()
    before = srv.pull(torch.arange(2 * keys, device="cuda"))[:, :dim]
    srv.muon_step(0, torch.cat([d_up, d_down]), 0.01)
    moved = srv.pull(torch.arange(2 * keys, device="cuda"))[:, :dim] - before
    grads = torch.cat([d_up, d_down]).view(2 * keys, dim)
    assert ((moved * grads).view(2 * experts, -1).sum(1) < 0).all()
    srv.status()
