"""Orthogonalised updates (muon_orthogonalize, muon_step) against the formulas in 64 bits: sides of one to a thousand, batches, types,
strides, matrices of zeros, of one direction, with infinities, of extreme magnitude; a step's momentum, weights and statistics; refusals.

Tolerance.  A step rounds X, A, P and their sums: relative errors of the unit u of the numbers (2^-24: 32-bit results, 2^-12: bf16 results) in a
handful of places - 8 are allowed -, relative to |X_k|_F.  What follows multiplies an error in a direction of singular value s by F(s) / s, F the
steps that are left; the largest of these quotients over the matrix's own singular values, and the limit at 0 where there are directions of none, is the gain.  So
|error|_F <= 8 u sum_k gain_k |X_k|_F, and half a unit of the result's own type for each element."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def p(s):
    return A * s + B * s ** 3 + C * s ** 5


def reference(d, steps=5, eps=1e-7, unit=2.0 ** -24):
    """The matrix orthogonalised, by its singular values, and what the products may be off by (Frobenius norm)."""
    d = d.astype(np.float64)
    norm = np.linalg.norm(d)
    if norm == 0.0:
        return np.zeros_like(d), 0.0
    u, s, vt = np.linalg.svd(d / (norm + eps), full_matrices=False)
    every = [s]
    for _ in range(steps):
        every.append(p(every[-1]))
    off = 0.0
    for k in range(steps):
        t, left = np.concatenate([[1e-9], np.maximum(every[k], 1e-9)]), steps - k
        x = t
        for _ in range(left):
            x = p(x)
        full = min(d.shape) > 1 or max(d.shape) > 1
        off += 8 * unit * float(np.max(np.abs(x / t)[0 if deficient(s) and full else 1:])) * float(np.linalg.norm(every[k]))
    return (u * every[-1]) @ vt, off


def deficient(s):
    return s.min() < 1e-4 * s.max()


def check(got, d, kind, unit, what, eps=1e-7):
    want, off = reference(d, unit=unit, eps=eps)
    err = np.linalg.norm(got.astype(np.float64) - want)
    tol = off + 1.01 * HALF[kind] * np.linalg.norm(want) + 1e-30
    print(f"  {what}: error {err / max(np.linalg.norm(want), 1e-300):.2e}, allowed {tol / max(np.linalg.norm(want), 1e-300):.2e}", flush=True)
    assert err <= tol, (what, err, tol)


@pytest.fixture(scope="module")
def srv():
    from paper_2002_00655_amd import ps as P
    return P.ParameterServer(1, 1, 1)


def gaussian(rng, *shape):
    return rng.standard_normal(shape).astype(np.float32)


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (3, 1, 7), (2, 5, 1), (4, 3, 3), (2, 16, 50), (1, 64, 64), (3, 65, 63), (16, 100, 100), (1, 127, 333), (2, 128, 128),
                                             (1, 129, 130), (2, 500, 70), (1, 70, 500), (1, 256, 1024), (1, 1030, 515), (5, 33, 257), (1, 1, 5000), (1, 5000, 2),
                                             (40, 200, 190), (3, 1100, 1200)])
def test_orthogonalize(srv, batch, rows, cols):
    import torch
    rng = np.random.default_rng(rows * 1000 + cols)
    for kind in ("float32", "bfloat16", "float16"):
        print(f"case {batch} x {rows} x {cols} {kind}", flush=True)
        x = torch.from_numpy(gaussian(rng, batch, rows, cols) * 3).cuda().to(getattr(torch, kind))
        for out_kind in {kind, "float32"}:
            got = srv.muon_orthogonalize(x, dtype=getattr(torch, out_kind))
            assert got.shape == x.shape and got.dtype == getattr(torch, out_kind)
            for i in range(min(batch, 4)):
                check(got[i].double().cpu().numpy(), x[i].double().cpu().numpy(), out_kind, 2.0 ** -12 if out_kind == "bfloat16" else 2.0 ** -24, f"{out_kind} {i}")
            assert torch.equal(srv.muon_orthogonalize(x, dtype=getattr(torch, out_kind)), got)


@pytest.mark.parametrize("batch,rows,cols", [(2, 3, 3), (3, 20, 20), (1, 128, 100), (2, 130, 140), (1, 90, 700), (1, 600, 200), (1, 1700, 1750), (1, 2300, 2000), (26, 1000, 1010)])
@pytest.mark.parametrize("steps", [1, 2, 3, 5])
def test_few_strong_directions_in_bfloat16(srv, batch, rows, cols, steps):
    """Up to four directions thirty times as strong as all others: the first steps raise the others by a factor of 3.4 each, and errors with
    them.  The result is at most twice as far from the true one as the true one rounded to bfloat16 is (a simulation of the roundings in 64
    bits gives 1.2 to 1.5 times; with numbers of 11 bits throughout it is five times)."""
    import torch
    rng = np.random.default_rng(rows + cols + steps)
    k = max(1, min(8, rows, cols) // 2)
    x = 30 * gaussian(rng, batch, rows, k) @ gaussian(rng, batch, k, cols) / np.sqrt(k) + gaussian(rng, batch, rows, cols)
    d = torch.from_numpy((x * 1e-3).astype(np.float32)).cuda().to(torch.bfloat16)
    got = srv.muon_orthogonalize(d, steps=steps)
    for i in range(min(batch, 2)):
        want = d[i].double()
        want = want / (torch.linalg.norm(want) + 1e-7)
        for _ in range(steps):
            a = want @ want.T
            want = A * want + (B * a + C * a @ a) @ want
        rounded, err = (float(torch.linalg.norm(t.double() - want) / torch.linalg.norm(want)) for t in (want.to(torch.bfloat16), got[i]))
        print(f"  {i}: error {err:.2e}, of rounding alone {rounded:.2e}", flush=True)
        assert err <= 2 * rounded + 2.0 ** -24, (i, err, rounded)


@pytest.mark.parametrize("batch,rows,cols", [(1, 64, 256), (2, 256, 64), (1, 65, 256), (1, 64, 257), (2, 10, 250), (3, 129, 64), (300, 30, 40), (1000, 64, 64), (257, 100, 128)])
def test_small_matrices_and_many_of_them(srv, batch, rows, cols):
    """At the limits of what one workgroup takes; batches by which larger matrices would be cut into larger tiles."""
    import torch
    rng = np.random.default_rng(batch + rows + cols)
    for kind in ("float32", "bfloat16"):
        x = torch.from_numpy(gaussian(rng, batch, rows, cols)).cuda().to(getattr(torch, kind))
        got = srv.muon_orthogonalize(x)
        for i in {0, batch // 2, batch - 1}:
            check(got[i].double().cpu().numpy(), x[i].double().cpu().numpy(), kind, 2.0 ** -12 if kind == "bfloat16" else 2.0 ** -24, f"{kind} {i}")


@pytest.mark.parametrize("rows,cols", [(1, 300), (2, 257), (4, 376), (700, 5), (8, 1000), (289, 11), (16, 2000), (33, 300), (600, 64)])
@pytest.mark.parametrize("strong", [1, 30])
def test_few_rows_in_bfloat16(srv, rows, cols, strong):
    """An error of one of a few numbers of P would be in a whole row of the result.  The numbers of the products are 2^-23 off, which is a thousandth of the
    result's rounding even where the steps raise it forty times: the result is within a fiftieth of the true one rounded."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows + cols + strong)
    d = (torch.randn(6, rows, cols, device="cuda", generator=g) + strong * torch.randn(6, rows, 1, device="cuda", generator=g) * torch.randn(6, 1, cols, device="cuda", generator=g))
    d = d.to(torch.bfloat16)
    got = srv.muon_orthogonalize(d)
    for i in range(6):
        x = d[i].double() / (torch.linalg.norm(d[i].double()) + 1e-7)
        for _ in range(5):
            a = x @ x.T
            x = A * x + (B * a + C * a @ a) @ x
        rounded, err = (float(torch.linalg.norm(t.double() - x) / torch.linalg.norm(x)) for t in (x.to(torch.bfloat16), got[i]))
        assert err <= 1.02 * rounded, (i, err, rounded)


@pytest.mark.parametrize("batch,rows,cols", [(1, 4096, 1024), (1, 1000, 4000), (1, 700, 6000), (6, 900, 640), (9, 370, 1200), (1, 1700, 1750), (8, 900, 1000)])
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
def test_millions_of_numbers(srv, batch, rows, cols, kind):
    """Tiles of 128 where there are fewer than compute units: sums over k that several workgroups share, and short ones, which go by tiles of 64."""
    import torch
    rng = np.random.default_rng(rows + cols)
    x = torch.from_numpy(gaussian(rng, batch, rows, cols)).cuda().to(getattr(torch, kind))
    got = srv.muon_orthogonalize(x)
    assert torch.equal(srv.muon_orthogonalize(x), got)
    for i in sorted({0, batch - 1}):
        check(got[i].double().cpu().numpy(), x[i].double().cpu().numpy(), kind, 2.0 ** -12 if kind == "bfloat16" else 2.0 ** -24, f"{kind} {i}")
        if kind == "bfloat16":                                                          # (the header's bound is nearer)
            want, _ = reference(x[i].double().cpu().numpy())
            assert np.linalg.norm(got[i].double().cpu().numpy() - want) <= 0.005 * np.linalg.norm(want)


@pytest.mark.parametrize("batch,rows,cols", [(1, 4096, 4096), (4, 2560, 2560), (2, 2300, 5100), (1, 4300, 4340), (8, 2048, 2048)])
@pytest.mark.parametrize("steps", [1, 2, 4, 6])
def test_on_both_sides_of_the_rule_for_the_largest_tiles(srv, batch, rows, cols, steps):
    """One direction 10^4 times the others, the bounds of test_dominated_matrices..."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows + steps)
    d = torch.randn(batch, rows, cols, device="cuda", generator=g) + 100 * rows ** 0.5 * torch.randn(batch, rows, 1, device="cuda", generator=g)
    got = srv.muon_orthogonalize(d, steps=steps, dtype=torch.bfloat16)
    for i in {0, batch - 1}:
        x = d[i].double() / (torch.linalg.vector_norm(d[i].double()) + 1e-7)
        for _ in range(steps):
            a = x @ x.T
            x = A * x + (B * a + C * a @ a) @ x
        err = float(torch.linalg.vector_norm(got[i].double() - x) / torch.linalg.vector_norm(x))
        print(f"  {i}: {err:.2e}", flush=True)
        assert err <= 0.005 + 2.0 ** -21 * A ** steps, (i, err)


@pytest.mark.parametrize("batch,rows,cols", [(2, 4352, 4300), (2, 4350, 4600), (1, 6100, 5888)])
def test_the_largest_tiles_through_five_steps(srv, batch, rows, cols):
    """Sides that tiles of 256 fill: single numbers and pairs one after the other, full rounds of the compute units and a rest whose sums are
    shared, both ways round.  At most a fifth further from the true result than that rounded to bfloat16 is."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows)
    d = torch.randn(batch, rows, cols, device="cuda", generator=g).to(torch.bfloat16)
    got = srv.muon_orthogonalize(d)
    for i in range(batch):
        x = d[i].double() / (torch.linalg.norm(d[i].double()) + 1e-7)
        for _ in range(5):
            a = x @ x.T
            x = A * x + (B * a + C * a @ a) @ x
        rounded, err = (float(torch.linalg.norm(t.double() - x) / torch.linalg.norm(x)) for t in (x.to(torch.bfloat16), got[i]))
        print(f"  {i}: error {err:.2e}, of rounding alone {rounded:.2e}", flush=True)
        assert err <= 1.2 * rounded, (i, err, rounded)


@pytest.mark.parametrize("batch,rows,cols,steps", [(1, 4300, 4340, 1), (2, 4340, 4300, 3), (1, 4100, 4400, 2)])
def test_large_matrices_in_bfloat16(srv, batch, rows, cols, steps):
    """A few directions a hundred times as strong as the others.  At most twice as far from the true result as that rounded to bfloat16 is."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows)
    d = (torch.randn(batch, rows, cols, device="cuda", generator=g) + 100 * torch.randn(batch, rows, 1, device="cuda", generator=g)).to(torch.bfloat16)
    got = srv.muon_orthogonalize(d, steps=steps)
    for i in range(batch):
        x = d[i].double() / (torch.linalg.norm(d[i].double()) + 1e-7)
        for _ in range(steps):
            a = x @ x.T
            x = A * x + (B * a + C * a @ a) @ x
        rounded, err = (float(torch.linalg.norm(t.double() - x) / torch.linalg.norm(x)) for t in (x.to(torch.bfloat16), got[i]))
        print(f"  {i}: error {err:.2e}, of rounding alone {rounded:.2e}", flush=True)
        assert err <= 2 * rounded, (i, err, rounded)


@pytest.mark.parametrize("batch,rows,cols", [(1, 80, 300), (1, 130, 140), (2, 400, 500), (4, 850, 900), (1, 4352, 4352)])
@pytest.mark.parametrize("steps", [3, 5, 7, 10])
@pytest.mark.parametrize("kind", ["bfloat16", "float32"])
def test_dominated_matrices_are_as_near_as_the_header_says(srv, batch, rows, cols, steps, kind):
    """One to 32 singular values 10^2 to 10^6 times all others: what a step's roundings leave in the weak directions is raised by 3.4 in every step that
    follows.  The bounds are the header's: 8 units of 2^-24 a step, as everywhere here, raised by all steps; and for bfloat16 0.005, where a simulation in
    64 bits of what single numbers cost, the result's own rounding included, gives 0.0024, 0.0039 and 0.0044 after three, five and seven steps."""
    import torch
    if rows > 1000 and kind == "float32":
        pytest.skip("the same kernels as the batch of 850 x 900")
    g = torch.Generator("cuda").manual_seed(rows + steps)
    rand = lambda *s: torch.randn(*s, device="cuda", dtype=torch.float64, generator=g)  # noqa: E731
    for k, ratio in ((1, 1e2), (32, 1e2), (1, 1e4), (4, 1e4), (1, 1e6), (4, 1e6), (32, 1e6)):
        d = rand(batch, rows, cols) / (rows ** 0.5 + cols ** 0.5)
        for i in range(batch):
            d[i] += ratio * (rand(rows, k) / rows ** 0.5) @ (rand(k, cols) / cols ** 0.5)
        d = d.float()
        got = srv.muon_orthogonalize(d, steps=steps, dtype=getattr(torch, kind))
        for i in range(min(batch, 2)):
            x = d[i].double()
            x = x / (torch.linalg.vector_norm(x) + 1e-7)
            for _ in range(steps):
                a = x @ x.T
                x = A * x + (B * a + C * a @ a) @ x
            err = float(torch.linalg.vector_norm(got[i].double() - x) / torch.linalg.vector_norm(x))
            print(f"  {k} by {ratio:g}: {err:.2e}", flush=True)
            assert err <= (0.005 if kind == "bfloat16" else 0.0) + 2.0 ** -21 * A ** steps, (k, ratio, i, err)


@pytest.mark.parametrize("rows,cols", [(60, 60), (200, 90), (90, 300), (1030, 1030)])
def test_every_matrix_of_a_batch_by_itself(srv, rows, cols):
    """Zeros, one direction, extreme magnitudes, infinities and NaN, side by side."""
    import torch
    rng = np.random.default_rng(rows)
    x = gaussian(rng, 7, rows, cols)
    x[0] = 0.0
    x[1] = np.outer(gaussian(rng, rows), gaussian(rng, cols))
    x[2] *= np.float32(1e-25)
    x[3] *= np.float32(1e25)
    x[4, rows // 2, cols // 3] = np.inf
    x[5, rows - 1, 0] = np.nan
    eps = 0.0 if rows == 60 else 1e-7
    got = srv.muon_orthogonalize(torch.from_numpy(x).cuda(), eps=eps).cpu().numpy()
    tiny = 1e-25 * np.sqrt(rows * cols)                                                 # its norm is far below 1e-7
    assert (got[0] == 0).all() or (rows == 60 and np.isnan(got[0]).all())               # 0 / 0 without eps
    check(got[1], x[1], "float32", 2.0 ** -24, "one direction", eps)
    if rows == 60:
        check(got[2], x[2], "float32", 2.0 ** -24, "tiny", eps)
    else:
        assert np.abs(got[2]).max() <= 500 * tiny / 1e-7
    check(got[3], x[3], "float32", 2.0 ** -24, "huge", eps)
    assert np.isnan(got[4]).all() and np.isnan(got[5]).all()
    check(got[6], x[6], "float32", 2.0 ** -24, "plain", eps)


@pytest.mark.parametrize("rows,cols", [(60, 60), (10, 300), (300, 100), (200, 190), (600, 600), (1800, 1700)])
@pytest.mark.parametrize("ratio", [1.0, 1e-3, 1e-6])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_matrices_whose_norm_is_below_eps(srv, rows, cols, ratio, kind):
    """X_0 is as small as |D| / eps, and every step raises it 3.4 times.  A step's roundings: 8 units of the numbers as everywhere here, relatively, and 2^-39 of
    each element, which the steps that are left raise; for bfloat16 the header's 0.005 beside that."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows)
    eps, steps = 1e-7, 5
    d = torch.randn(2, rows, cols, device="cuda", dtype=torch.float64, generator=g)
    d = (d / torch.linalg.vector_norm(d, dim=(1, 2), keepdim=True) * (eps * ratio)).float()
    got = srv.muon_orthogonalize(d, eps=eps, dtype=getattr(torch, kind))
    for i in range(2):
        x = d[i].double() / (torch.linalg.vector_norm(d[i].double()) + np.float64(np.float32(eps)))
        off = 0.0
        for k in range(steps):
            left = A ** (steps - k)
            off += left * (2.0 ** -21 * float(torch.linalg.vector_norm(x)) + 2.0 ** -39 * (rows * cols) ** 0.5)
            a = x @ x.T
            x = A * x + (B * a + C * a @ a) @ x
        norm = float(torch.linalg.vector_norm(x))
        err = float(torch.linalg.vector_norm(got[i].double() - x))
        off += (0.005 if kind == "bfloat16" else 2.0 ** -24) * norm
        print(f"  {i}: error {err / norm:.2e}, allowed {off / norm:.2e}", flush=True)
        assert err <= off, (i, err, off)


@pytest.mark.parametrize("batch,rows,cols", [(2, 1, 1), (3, 60, 60), (2, 10, 300), (3, 300, 100), (2, 200, 190), (4, 850, 900), (2, 4352, 4352)])
@pytest.mark.parametrize("eps", [0.0, 1e-7])
def test_a_matrix_of_zeros_stays_zero(srv, batch, rows, cols, eps):
    """Beside one that does not, and in the step: weights whose gradient and momentum are zero only decay."""
    import torch
    g = torch.Generator("cuda").manual_seed(rows)
    x = torch.randn(batch, rows, cols, device="cuda", generator=g)
    x[0] = 0
    for kind in (torch.float32, torch.bfloat16):
        got = srv.muon_orthogonalize(x, eps=eps, dtype=kind)
        assert (got[0] == 0).all() and torch.isfinite(got[1:].float()).all() and (got[1:] != 0).any()
    if cols <= 512:
        w = torch.randn(rows, 2 * cols, device="cuda", generator=g)
        w[:, cols:] = 0
        s = server(w.cpu().numpy())
        s.muon_step(0, torch.zeros(rows, cols, device="cuda"), 0.5, weight_decay=0.25, eps=eps)
        w[:, :cols] *= 0.875
        assert torch.equal(s.pull(torch.arange(rows, device="cuda")), w)


@pytest.mark.parametrize("steps", [1, 2, 5, 9])
def test_number_of_steps(srv, steps):
    import torch
    rng = np.random.default_rng(steps)
    x = gaussian(rng, 80, 120)
    got = srv.muon_orthogonalize(torch.from_numpy(x).cuda(), steps=steps).cpu().numpy()
    want, off = reference(x, steps=steps)
    assert np.linalg.norm(got - want) <= off + 2.0 ** -24 * np.linalg.norm(want)


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_strided_matrices(srv, kind):
    """Rows at any distance and alignment; what lies between the rows of the result stays."""
    import torch
    rng = np.random.default_rng(1)
    dt = getattr(torch, kind)
    for rows, cols, gap, offset in ((70, 130, 3, 1), (130, 70, 6, 2), (64, 64, 0, 3), (33, 10, 1, 0)):
        base = torch.from_numpy(gaussian(rng, 2 * rows * (cols + gap) + offset + cols)).cuda().to(dt)
        view = base[offset:].as_strided((2, rows, cols), (rows * (cols + gap), cols + gap, 1))
        to = torch.full_like(base, 7.0)
        out = to[offset:].as_strided((2, rows, cols), (rows * (cols + gap), cols + gap, 1))
        want = srv.muon_orthogonalize(view.contiguous())
        assert srv.muon_orthogonalize(view, out=out) is out and torch.equal(out, want)
        out.fill_(7.0)
        assert (to == 7.0).all()


@pytest.mark.parametrize("rows,cols", [(60, 60), (300, 40), (300, 130)])
def test_expanded_matrices(srv, rows, cols):
    """Gradients as sums pass them back: one number, a number of each row, or a row for all; of two and three dimensions."""
    import torch
    rng = np.random.default_rng(rows + cols)
    col, row, number = (torch.from_numpy(gaussian(rng, *s)).cuda() for s in ((rows, 1), (1, cols), ()))
    a, b = server(np.ones((2 * rows, 2 * cols), np.float32)), server(np.ones((2 * rows, 2 * cols), np.float32))
    for x in (number.expand(rows, cols), col.expand(rows, cols), row.expand(rows, cols)):
        for d in (x, x.expand(2, rows, cols)):
            assert torch.equal(srv.muon_orthogonalize(d), srv.muon_orthogonalize(d.contiguous()))
            a.muon_step(0, d, 0.1)
            b.muon_step(0, d.contiguous(), 0.1)
    keys = torch.arange(2 * rows, device="cuda")
    assert torch.equal(a.pull(keys), b.pull(keys))
    with pytest.raises(ValueError):
        srv.muon_orthogonalize(col.expand(rows, cols), out=torch.zeros(rows, 1, device="cuda").expand(rows, cols))


def server(values, W=1):
    import torch
    from paper_2002_00655_amd import ps as P
    s = P.ParameterServer(values.shape[0], values.shape[1], W)
    s.push(torch.arange(values.shape[0], device="cuda"), torch.from_numpy(values).cuda())
    return s


@pytest.mark.parametrize("batch,rows,dim,L,first,kind", [(1, 1, 1, 2, 0, "float32"), (1, 333, 127, 254, 0, "float32"), (3, 40, 64, 130, 9, "bfloat16"), (2, 100, 100, 200, 1, "float16"),
                                                         (1, 700, 512, 1024, 3, "bfloat16"), (4, 30, 300, 601, 0, "float32"), (1, 17, 5, 10, 100, "bfloat16")])
def test_step(batch, rows, dim, L, first, kind):
    import torch
    rng = np.random.default_rng(rows + dim)
    print(f"case {batch} x {rows} x {dim} {kind}", flush=True)
    keys = batch * rows
    values = gaussian(rng, first + keys + 5, L) * np.float32(0.05)
    srv = server(values)
    lr, wd, mu = 0.02, 0.1, 0.9
    f = lambda v: float(np.float32(v))  # noqa: E731  (what the call gets)
    want, tol = values.astype(np.float64), np.zeros(keys)
    W, M = want[first:first + keys, :dim], want[first:first + keys, dim:2 * dim]
    off = 0.0
    for it in range(3):
        nesterov = it != 1
        grad = torch.from_numpy(gaussian(rng, batch, rows, dim)).cuda().to(getattr(torch, kind))
        srv.muon_step(first, grad, lr, momentum=mu, nesterov=nesterov, weight_decay=wd)
        g = grad.double().cpu().numpy().reshape(keys, dim)
        M[:] = f(mu) * M + g
        d = g + f(mu) * M if nesterov else M
        step = f(lr) * np.sqrt(max(1.0, rows / dim))
        W *= 1 - f(lr) * f(wd)
        for i in range(batch):
            o, e = reference(d[i * rows:(i + 1) * rows])
            W[i * rows:(i + 1) * rows] -= step * o
            off += step * e
        off += 8 * 2.0 ** -24 * (np.linalg.norm(W) + step * np.sqrt(batch * min(rows, dim)))
        got = srv.pull(torch.arange(first + keys + 5, device="cuda")).cpu().numpy()
        at = slice(first, first + keys)
        assert np.linalg.norm(got[at, :dim] - W) <= off, (np.linalg.norm(got[at, :dim] - W), off)
        assert np.abs(got[at, dim:2 * dim] - M).max() <= 4 * (it + 1) * 2.0 ** -24 * max(1.0, np.abs(M).max())
        rest = np.ones(values.shape, bool)
        rest[at, :2 * dim] = False
        assert np.array_equal(got[rest], values[rest])
    srv.status()


@pytest.mark.parametrize("batch,rows,dim,L,first,kind", [(8, 2048, 512, 1024, 2, "bfloat16"), (5, 1500, 471, 943, 7, "float32"), (20, 300, 500, 1001, 1, "float16"),
                                                         (12, 471, 500, 1000, 0, "bfloat16")])
def test_step_of_many_numbers(batch, rows, dim, L, first, kind):
    """Batches that are cut into tiles of 128: more of them than compute units and fewer, sums that are shared, sums that are short; rows of the server that
    cannot be written eight numbers at a time.  Tolerances as in test_step."""
    import torch
    rng = np.random.default_rng(rows + dim)
    print(f"case {batch} x {rows} x {dim} {kind}", flush=True)
    keys = batch * rows
    values = gaussian(rng, first + keys + 3, L) * np.float32(0.05)
    srv = server(values)
    lr, wd, mu = 0.02, 0.1, 0.9
    f = lambda v: float(np.float32(v))  # noqa: E731
    grad = torch.from_numpy(gaussian(rng, batch, rows, dim)).cuda().to(getattr(torch, kind))
    srv.muon_step(first, grad, lr, momentum=mu, nesterov=True, weight_decay=wd)
    got = srv.pull(torch.arange(first + keys + 3, device="cuda")).cpu().numpy()
    g = grad.double().cpu().numpy().reshape(keys, dim)
    at, step = slice(first, first + keys), f(lr) * np.sqrt(max(1.0, rows / dim))
    M = f(mu) * values[at, dim:2 * dim].astype(np.float64) + g
    for i in sorted({0, 1, batch // 2, batch - 1}):
        r = slice(i * rows, (i + 1) * rows)
        o, off = reference(g[r] + f(mu) * M[r])
        W = (1 - f(lr) * f(wd)) * values[at, :dim][r].astype(np.float64) - step * o
        tol = step * off + 8 * 2.0 ** -24 * (np.linalg.norm(W) + step * np.sqrt(min(rows, dim)))
        err = np.linalg.norm(got[at, :dim][r] - W)
        print(f"  {i}: error {err:.2e}, allowed {tol:.2e}", flush=True)
        assert err <= tol, (i, err, tol)
    assert np.abs(got[at, dim:2 * dim] - M).max() <= 4 * 2.0 ** -24 * max(1.0, np.abs(M).max())
    rest = np.ones(values.shape, bool)
    rest[at, :2 * dim] = False
    assert np.array_equal(got[rest], values[rest])
    srv.status()


def test_step_statistics_and_a_standing_error():
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(2)
    K, L, W = 300, 32, 4
    values = gaussian(rng, K, L)
    for caches in (0, 1):
        a, b = server(values, W), server(values, W)
        for s in (a, b):
            s.set_option(P.OPT_LOCATION_CACHES, caches)
            s.localize(torch.arange(0, K, 2, device="cuda"), 3)
        for worker in (-1, 0, 3, 3, 0):
            grad = torch.from_numpy(gaussian(rng, 2, 100, 16)).cuda()
            keys = torch.arange(40, 240, device="cuda")
            a.muon_step(40, grad, 0.01, worker=worker)
            b.pull(keys, worker)
            b.push(keys, torch.zeros(200, L, device="cuda"), worker)
            assert a.stats() == b.stats()
        # a call before it named a key that is not there: nothing is changed until the status has been asked for
        before, stats = a.pull(torch.arange(K, device="cuda")), a.stats()
        a.pull(torch.tensor([K], device="cuda"))
        a.muon_step(40, grad, 0.01, worker=1)
        with pytest.raises(P.PSError):
            a.status()
        assert torch.equal(a.pull(torch.arange(K, device="cuda")), before) and a.stats() == stats


def test_empty_batches_and_refusals(srv):
    import torch
    from paper_2002_00655_amd import ps as P
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    for shape in ((0, 4, 4), (3, 0, 4), (3, 4, 0)):
        assert srv.muon_orthogonalize(z(*shape)).shape == shape
    s = server(np.ones((100, 16), np.float32), W=2)
    s.muon_step(0, z(0, 10, 8), 0.1)
    s.muon_step(100, z(1, 0, 8), 0.1)
    for code, call in ((P.PS_EINVAL, lambda: srv.muon_orthogonalize(z(4, 4), steps=0)), (P.PS_EINVAL, lambda: srv.muon_orthogonalize(z(4, 4), steps=101)),
                       (P.PS_EINVAL, lambda: srv.muon_orthogonalize(z(4, 4), eps=-1.0)), (P.PS_EINVAL, lambda: srv.muon_orthogonalize(z(4, 4), eps=float("nan"))),
                       (P.PS_ELIMIT, lambda: srv.muon_orthogonalize(z(1, 32769))), (P.PS_ELIMIT, lambda: srv.muon_orthogonalize(z(65536, 1, 1))),
                       (P.PS_EINVAL, lambda: s.muon_step(0, z(10, 9), 0.1)), (P.PS_EINVAL, lambda: s.muon_step(91, z(10, 8), 0.1)),
                       (P.PS_EINVAL, lambda: s.muon_step(-1, z(10, 8), 0.1)), (P.PS_EWORKER, lambda: s.muon_step(0, z(10, 8), 0.1, worker=2)),
                       (P.PS_EINVAL, lambda: s.muon_step(0, z(10, 8), 0.1, steps=0)), (P.PS_EINVAL, lambda: s.muon_step(0, z(101, 1, 8), 0.1))):
        with pytest.raises(P.PSError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: srv.muon_orthogonalize(z(4, 4).double()), lambda: srv.muon_orthogonalize(torch.zeros(4, 4)), lambda: srv.muon_orthogonalize(z(4, 4), dtype=torch.float64)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: srv.muon_orthogonalize(z(4)), lambda: srv.muon_orthogonalize(z(4, 5).t()), lambda: srv.muon_orthogonalize(z(4, 4), out=z(4, 5)),
                 lambda: srv.muon_orthogonalize(z(4, 3, 5), out=z(3, 4, 5).transpose(0, 1))):
        with pytest.raises(ValueError):
            call()
    assert (s.pull(torch.arange(100, device="cuda")) == 1).all()


def test_on_another_stream_and_in_a_graph(srv):
    import torch
    rng = np.random.default_rng(7)
    values = gaussian(rng, 200, 64)
    a, b = server(values), server(values)
    x, out, grad = torch.zeros(3, 70, 90, device="cuda"), torch.zeros(3, 70, 90, device="cuda"), torch.zeros(2, 100, 32, device="cuda")

    def calls(s):
        s.muon_orthogonalize(x, out=out)
        s.muon_step(0, grad, 0.02, weight_decay=0.1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(a)
    torch.cuda.current_stream().wait_stream(side)
    calls(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(a)
    for _ in range(3):
        x.copy_(torch.from_numpy(gaussian(rng, 3, 70, 90)))
        grad.copy_(torch.from_numpy(gaussian(rng, 2, 100, 32)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        calls(b)
        keys = torch.arange(200, device="cuda")
        assert torch.equal(got, out) and torch.equal(a.pull(keys), b.pull(keys))
