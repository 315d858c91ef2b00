"""Tokens (emb_lookup, emb_grad, emb_adagrad_step) against the formulas in 64 bits: types, row lengths, strides and alignments,
one token to many, padding, tokens of all rows and of one, rows of a table in a larger server; refusals and bad tokens.

Tolerances, relative to the sum of the absolute values that go into a result: a sum of m terms in 32 bits, in ranges of up to 64 and over
the ranges, has at most (64 + m / 8) roundings behind each other, of 2^-24 each; in practice the root of that."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
ROUND = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}      # half a unit of 24, 8 and 11 bits, relative


def _server(K, L, W=1, seed=0):
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(seed)
    values = rng.standard_normal((K, L)).astype(np.float32)
    values[:, L // 2:] = np.abs(values[:, L // 2:])
    srv = P.ParameterServer(K, L, W)
    srv.push(torch.arange(K, device="cuda"), torch.from_numpy(values).cuda())
    return srv, values


def _all(srv):
    import torch
    return srv.pull(torch.arange(srv.K, device="cuda")).cpu().numpy()


def _close(got, want, scale, rel):
    """|got - want| <= rel * scale, element by element (and a little for numbers that the type cannot hold exactly near zero)"""
    err = np.abs(got.astype(np.float64) - want)
    bad = err > rel * scale + 6.0e-8 * (rel > 2.0 ** -12)
    assert not bad.any(), (int(bad.sum()), float((err / np.maximum(scale, 1e-300)).max()), rel)


def _sums(tokens, dout, V, pad):
    keep = tokens != pad if pad is not None else np.ones(tokens.size, bool)
    want, mag = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    np.add.at(want, tokens[keep], dout[keep])
    np.add.at(mag, tokens[keep], np.abs(dout[keep]))
    return want, mag, np.bincount(tokens[keep], minlength=V)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 2048, 2049, 5000])
@pytest.mark.parametrize("K,L,dim,first", [(700, 128, 128, 0), (300, 100, 50, 20), (97, 51, 51, 7), (64, 1024, 512, 0), (50, 1, 1, 3), (40, 1022, 1022, 0)])
def test_lookup(n, K, L, dim, first):
    import torch
    print(f"case n={n} K={K} L={L} dim={dim}", flush=True)
    rng = np.random.default_rng(n + L)
    srv, values = _server(K, L)
    V = K - first - 2
    for kind in TYPES:
        for wide in (False, True):
            for pad in (None, 0, -100):
                tokens = rng.integers(0, V, size=n)
                if pad is not None:
                    tokens[rng.random(n) < 0.4] = pad
                t = torch.from_numpy(tokens.astype(np.int64 if wide else np.int32)).cuda()
                got = srv.emb_lookup(t, first_key=first, num_tokens=V, dim=dim, scale=3.7, pad_token=pad, dtype=getattr(torch, kind))
                want = values.astype(np.float64)[np.maximum(tokens, 0) + first, :dim] * np.float64(np.float32(3.7))
                if pad is not None:
                    want[tokens == pad] = 0.0
                _close(got.float().cpu().numpy(), want, np.abs(want), 2.0 ** -24 + ROUND[kind] * (kind != "float32"))
    srv.status()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("offset,gap", [(0, 0), (1, 0), (0, 3), (2, 6), (4, 4), (8, 8)])
def test_lookup_into_strided_rows(kind, offset, gap):
    """Rows at any distance and alignment; what lies between them stays."""
    import torch
    rng = np.random.default_rng(offset + gap)
    srv, values = _server(90, 64)
    tokens = torch.from_numpy(rng.integers(0, 90, size=(5, 7))).cuda()
    base = torch.full((35 * (64 + gap) + offset + 64,), 7.0, device="cuda", dtype=getattr(torch, kind))
    out = base[offset:].as_strided((5, 7, 64), (7 * (64 + gap), 64 + gap, 1))
    assert srv.emb_lookup(tokens, out=out) is out
    assert torch.equal(out, torch.from_numpy(values).cuda()[tokens].to(out.dtype))
    left = base.clone()
    left[offset:].as_strided((5, 7, 64), (7 * (64 + gap), 64 + gap, 1)).fill_(7.0)
    assert (left == 7.0).all()


def test_lookup_passes_infinities_and_nan_and_no_padding_row():
    import torch
    srv, _ = _server(10, 8)
    srv.push(torch.tensor([3, 4], device="cuda"), torch.tensor([[float("inf")] * 8, [float("nan")] * 8], device="cuda"))
    out = srv.emb_lookup(torch.tensor([3, 4, 5], device="cuda"), pad_token=4, dtype=torch.bfloat16)
    assert torch.isinf(out[0]).all() and (out[1] == 0).all() and torch.isfinite(out[2].float()).all()


@pytest.mark.parametrize("n", [0, 1, 2, 7, 64, 65, 130, 2048, 2049, 9000, 70_000])
@pytest.mark.parametrize("V,D", [(1, 4), (37, 64), (900, 100), (5000, 51), (300, 512), (2000, 260), (40, 1030), (70_001, 8)])
def test_gradient(n, V, D):
    import torch
    from paper_2002_00655_amd import ps as P
    if n * D > 20_000_000:
        n = 20_000_000 // D
    print(f"case n={n} V={V} D={D}", flush=True)
    rng = np.random.default_rng(n + V + D)
    srv = P.ParameterServer(1, 1, 1)
    for i, kind in enumerate(TYPES):
        pad = (None, V // 2, -1)[i]
        tokens = np.minimum((V * rng.random(n) ** 3).astype(np.int64), V - 1)           # the first ones often
        if pad is not None:
            tokens[rng.random(n) < 0.2] = pad
        dout = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).cuda().to(getattr(torch, kind))
        t = torch.from_numpy(tokens.astype(np.int32 if i % 2 else np.int64)).cuda()
        want, mag, count = _sums(tokens, dout.double().cpu().numpy(), V, pad)
        tol = (64 + count / 8 + 3)[:, None] * 2.0 ** -24
        scale = np.float64(np.float32(0.3))
        got = srv.emb_grad(t, dout, V, scale=0.3, pad_token=pad, grad=torch.full((V, D), 9.0, device="cuda"))
        _close(got.cpu().numpy(), want * scale, mag * scale, tol)
        assert (got.cpu().numpy()[count == 0] == 0.0).all()
        had = torch.from_numpy(rng.standard_normal((V, D)).astype(np.float32)).cuda()
        more = srv.emb_grad(t, dout, V, scale=0.3, pad_token=pad, grad=had.clone(), accumulate=True)
        assert torch.equal(more, torch.where(torch.from_numpy(count == 0).cuda()[:, None], had, had + got))
        again = srv.emb_grad(t, dout, V, scale=0.3, pad_token=pad)
        assert torch.equal(again, got)
    srv.status()


@pytest.mark.parametrize("n", [2049, 2112, 4095, 4096, 4097, 8128, 8191, 8192, 8193, 16_385, 131_073, 262_145])
def test_every_term_is_added_once_whatever_sorts_the_tokens(n):
    """Sums of small integers are exact, in any order: how often a token comes, and at which positions."""
    import torch
    from paper_2002_00655_amd import ps as P
    srv = P.ParameterServer(1, 1, 1)
    rng = np.random.default_rng(n)
    for V, pad, wide in ((1, None, True), (130, 129, False), (70_000, 0, True), (100_000, -5, False)):
        tokens = rng.integers(0, V, n)
        if pad is not None:
            tokens[rng.random(n) < 0.1] = pad
        dout = np.stack([np.ones(n), np.arange(n) % 8, np.arange(n) // 8 % 8], 1).astype(np.float32)
        got = srv.emb_grad(torch.from_numpy(tokens.astype(np.int64 if wide else np.int32)).cuda(), torch.from_numpy(dout).cuda(), V, pad_token=pad).cpu().numpy()
        there = tokens != pad if pad is not None else np.ones(n, bool)
        for c in range(3):
            assert np.array_equal(got[:, c], np.bincount(tokens[there], weights=dout[there, c], minlength=V).astype(np.float32)), (V, c)


@pytest.mark.parametrize("n", [262_144, 2_097_152, 2_097_153, 5_000_001])
@pytest.mark.parametrize("V,pad,wide", [(1, None, True), (2, None, False), (130, 129, False), (100_000, -5, True), (70_000_000, 0, False)])
def test_every_term_is_added_once_of_millions(n, V, pad, wide):
    """As above, up to the tiles of the longest sorts; sums stay below 2^24.  One token or two: one workgroup joins all ranges."""
    import torch
    from paper_2002_00655_amd import ps as P
    print(f"case n={n} V={V}", flush=True)
    g = torch.Generator("cuda").manual_seed(n + V)
    tokens = torch.randint(0, V, (n,), device="cuda", generator=g)
    if pad is not None:
        tokens[torch.rand(n, device="cuda", generator=g) < 0.1] = pad
    q = torch.arange(n, device="cuda")
    dout = torch.stack([torch.ones_like(q), q % 2, q // 2 % 3 // 2], 1).float()
    srv = P.ParameterServer(1, 1, 1)
    got = srv.emb_grad(tokens if wide else tokens.int(), dout, V, pad_token=pad)
    there = tokens != pad if pad is not None else torch.ones_like(tokens, dtype=torch.bool)
    for c in range(3):
        want = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, tokens[there], dout[there, c].double())
        assert torch.equal(got[:, c].double(), want), c
    srv.status()


def test_offsets_past_32_bits():
    """A result, a gradient of the result and a server of more than 2^31 numbers: their last rows."""
    import torch
    from paper_2002_00655_amd import ps as P
    # the result: 4,300,000 rows of 512
    rng, n = np.random.default_rng(0), 4_300_000
    srv, values = _server(900, 512)
    rows = torch.from_numpy(values).cuda()
    tokens = torch.randint(0, 900, (n,), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    out = srv.emb_lookup(tokens, dtype=torch.bfloat16)
    for a in (0, n // 2, 4_194_300, n - 1000):                                             # (the 4,194,304th row starts at number 2^31)
        assert torch.equal(out[a:a + 1000], rows[tokens[a:a + 1000]].to(torch.bfloat16))
    # its gradient, every 500th row of it
    out.zero_()
    some = torch.arange(0, n, 500, device="cuda")
    dout = out[::500]
    dout.copy_(torch.from_numpy(rng.integers(-8, 9, size=(some.numel(), 512)).astype(np.float32)))
    want = torch.zeros(900, 512, dtype=torch.float64, device="cuda").index_add_(0, tokens[some], dout.double())
    assert dout.stride(0) * (some.numel() - 1) > 1 << 31 and torch.equal(srv.emb_grad(tokens[some], dout, 900).double(), want)
    del out, dout, srv
    # the server: 2,200,000 keys of 1,024
    K, first = 2_200_000, 2_100_000
    srv = P.ParameterServer(K, 1024, 1)
    keys = torch.arange(first - 5, K, device="cuda")
    at = torch.randint(0, K - first, (3000,), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    was = torch.rand(keys.numel(), 1024, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    srv.push(keys, was)
    assert torch.equal(srv.emb_lookup(at, first_key=first), was[5 + at])
    srv.emb_adagrad_step(at, torch.ones(3000, 512, device="cuda"), 0.5, 1.0, first_key=first)
    got, count = srv.pull(keys), torch.bincount(at, minlength=K - first)
    hit = torch.cat([torch.zeros(5, device="cuda"), count.float()])[:, None]
    acc = was[:, 512:] + hit * hit
    assert torch.equal(got[:, 512:], acc)
    want = was[:, :512].double() - 0.5 * hit.double() / torch.sqrt(acc.double() + 1.0)
    assert float((got[:, :512].double() - want).abs().max()) <= 4 * 2.0 ** -24
    same = hit[:, 0] == 0
    assert torch.equal(got[same], was[same])
    srv.status()


@pytest.mark.parametrize("n", [2052, 4096, 4100, 8192, 8196, 131_072, 131_076])
def test_terms_are_added_in_the_order_of_their_positions(n):
    """Four terms a token, which lie in one range: the sums are those of 32-bit additions one after the other, bit for bit."""
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(n)
    tokens = rng.permutation(np.repeat(np.arange(n // 4), 4))
    dout = rng.standard_normal((n, 5)).astype(np.float32)
    got = P.ParameterServer(1, 1, 1).emb_grad(torch.from_numpy(tokens).cuda(), torch.from_numpy(dout).cuda(), n // 4).cpu().numpy()
    d = dout[np.argsort(tokens, kind="stable")].reshape(n // 4, 4, 5)
    assert np.array_equal(got, ((d[:, 0] + d[:, 1]) + d[:, 2]) + d[:, 3])


@pytest.mark.parametrize("n", [0, 100, 3000])
def test_gradient_of_a_vocabulary_of_many_millions(n):
    """More rows to clear than one workgroup each takes; the rest of a row of one number."""
    import torch
    from paper_2002_00655_amd import ps as P
    V = 70_000_013
    rng = np.random.default_rng(n)
    tokens = rng.choice(V, n, replace=False) if n else np.zeros(0, np.int64)
    tokens[:2] = (0, V - 1) if n else ()
    dout = rng.standard_normal((n, 1)).astype(np.float32)
    got = P.ParameterServer(1, 1, 1).emb_grad(torch.from_numpy(tokens).cuda(), torch.from_numpy(dout).cuda(), V, grad=torch.full((V, 1), 9.0, device="cuda"))
    want = torch.zeros(V, 1, device="cuda").index_add_(0, torch.from_numpy(tokens).cuda(), torch.from_numpy(dout).cuda())
    assert torch.equal(got, want)


@pytest.mark.parametrize("what", ["one token", "all padding", "every token once", "two tokens in turn"])
@pytest.mark.parametrize("n,D", [(65, 16), (4096, 128), (30_000, 72)])
def test_gradient_of_extreme_batches(what, n, D):
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(n)
    V = n + 3
    tokens = {"one token": np.full(n, 5), "all padding": np.full(n, 1), "every token once": rng.permutation(n), "two tokens in turn": np.arange(n) % 2 * 7}[what]
    pad = 1 if what == "all padding" else None
    dout = rng.standard_normal((n, D)).astype(np.float32)
    got = P.ParameterServer(1, 1, 1).emb_grad(torch.from_numpy(tokens).cuda(), torch.from_numpy(dout).cuda(), V, pad_token=pad).cpu().numpy()
    want, mag, count = _sums(tokens, dout.astype(np.float64), V, pad)
    _close(got, want, mag, (64 + count / 8 + 3)[:, None] * 2.0 ** -24)
    if what == "every token once":
        assert np.array_equal(got[tokens], dout)


def test_gradient_of_padding_is_ignored_whatever_it_holds():
    import torch
    from paper_2002_00655_amd import ps as P
    tokens = torch.tensor([2, 0, 2, 0, 1], device="cuda", dtype=torch.int32)
    dout = torch.ones(5, 12, device="cuda")
    dout[1], dout[3] = float("nan"), float("inf")
    got = P.ParameterServer(1, 1, 1).emb_grad(tokens, dout, 3, pad_token=0)
    assert torch.equal(got, torch.tensor([0.0, 1.0, 2.0], device="cuda")[:, None].expand(3, 12))


@pytest.mark.parametrize("kind", TYPES)
def test_gradient_of_broadcast_strided_and_misaligned_rows(kind):
    import torch
    from paper_2002_00655_amd import ps as P
    rng, srv = np.random.default_rng(5), P.ParameterServer(1, 1, 1)
    dt = getattr(torch, kind)
    for D in (64, 96, 512):
        tokens = torch.from_numpy(rng.integers(0, 50, size=(30, 11))).cuda()
        one = torch.from_numpy(rng.integers(-8, 9, size=D).astype(np.float32)).cuda().to(dt)
        count = torch.bincount(tokens.flatten(), minlength=50).float()
        assert torch.equal(srv.emb_grad(tokens, one.expand(30, 11, D), 50), count[:, None] * one.float())
        for offset, gap in ((0, 8), (1, 0), (3, 5)):
            base = torch.from_numpy(rng.integers(-8, 9, size=330 * (D + gap) + offset + D).astype(np.float32)).cuda().to(dt)
            rows = base[offset:].as_strided((30, 11, D), (11 * (D + gap), D + gap, 1))
            want = torch.zeros(50, D, device="cuda", dtype=torch.float64).index_add_(0, tokens.flatten(), rows.reshape(330, D).double())
            assert torch.equal(srv.emb_grad(tokens, rows, 50).double(), want)           # (integers: exact in any order)
        # rows that lie at no one distance
        rows = torch.from_numpy(rng.integers(-8, 9, size=(11, 30, D)).astype(np.float32)).cuda().to(dt).transpose(0, 1)
        want = torch.zeros(50, D, device="cuda", dtype=torch.float64).index_add_(0, tokens.flatten(), rows.reshape(330, D).double())
        assert torch.equal(srv.emb_grad(tokens, rows, 50).double(), want)


@pytest.mark.parametrize("n", [1, 60, 3000])
def test_gradient_of_expanded_numbers(n):
    """What a sum of a lookup's output, or of its rows' sums, passes back: strides of 0."""
    import torch
    from paper_2002_00655_amd import ps as P
    rng, D = np.random.default_rng(n), 36
    tokens = torch.from_numpy(rng.integers(0, 50, size=n)).cuda()
    srv, _ = _server(50, 2 * D)
    ref, _ = _server(50, 2 * D)
    row = torch.from_numpy(rng.integers(-8, 9, size=(n, 1)).astype(np.float32)).cuda()
    for dout in (torch.full((), 2.0, device="cuda").expand(n, D), row.expand(n, D), row[:1, :1].to(torch.bfloat16).expand(n, D)):
        want = srv.emb_grad(tokens, dout.contiguous(), 50)
        assert torch.equal(srv.emb_grad(tokens, dout, 50), want)
        if n == 60:
            assert torch.equal(srv.emb_grad(tokens.view(5, 12), dout.view(5, 12, D) if dout.stride(0) else dout[:1].expand(60, D).reshape(5, 12, D), 50), want)
        srv.emb_adagrad_step(tokens, dout, 0.1, 1e-8)
        ref.emb_adagrad_step(tokens, dout.contiguous(), 0.1, 1e-8)
    out = torch.full((), 3.0, device="cuda").expand(5, 12, D)
    assert torch.equal(srv.emb_grad(tokens[:1].expand(60).contiguous().view(5, 12), out, 50), srv.emb_grad(tokens[:1].expand(60).contiguous(), out.reshape(60, D).contiguous(), 50))
    assert np.array_equal(_all(srv), _all(ref))
    with pytest.raises(ValueError):
        srv.emb_lookup(tokens[:1].expand(7).contiguous(), dim=D, out=torch.zeros(7, 1, device="cuda").expand(7, D))
    srv.status()


def test_gradient_against_differences():
    """<dout, lookup(E + h X) - lookup(E - h X)> / 2h = <grad, X>: the lookup is linear, so no more than roundings."""
    import torch
    rng = np.random.default_rng(0)
    V, D, n, h = 60, 24, 500, 0.5
    a, va = _server(V, D, seed=1)
    x = rng.standard_normal((V, D)).astype(np.float32)
    tokens = torch.from_numpy(rng.integers(0, V, size=n)).cuda()
    dout = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).cuda()
    keys, dx = torch.arange(V, device="cuda"), torch.from_numpy(x).cuda()
    a.push(keys, h * dx)
    up = a.emb_lookup(tokens, scale=1.5, pad_token=4).double()
    a.push(keys, -2 * h * dx)
    down = a.emb_lookup(tokens, scale=1.5, pad_token=4).double()
    grad = a.emb_grad(tokens, dout, V, scale=1.5, pad_token=4).double()
    left, right = float((dout.double() * (up - down)).sum() / (2 * h)), float((grad * dx.double()).sum())
    size = float((dout.double() * up).abs().sum())
    assert abs(left - right) <= size * 2.0 ** -22, (left, right)


@pytest.mark.parametrize("n", [0, 1, 3, 64, 65, 2048, 2049, 20_000])
@pytest.mark.parametrize("V,D,L,first", [(50, 64, 128, 0), (333, 25, 51, 11), (4000, 128, 300, 5), (700, 512, 1024, 0), (9, 1, 2, 0)])
def test_adagrad_step(n, V, D, L, first):
    import torch
    print(f"case n={n} V={V} D={D} L={L}", flush=True)
    rng = np.random.default_rng(n + V)
    K = first + V + 4
    srv, values = _server(K, L, seed=n)
    values[:, D:2 * D] = np.abs(values[:, D:2 * D])
    srv2, _ = _server(1, 1)
    import paper_2002_00655_amd.ps as P
    srv = P.ParameterServer(K, L, 1)
    srv.push(torch.arange(K, device="cuda"), torch.from_numpy(values).cuda())
    want = values.astype(np.float64)
    err = np.zeros_like(want)
    lr, eps = 0.1, 1e-6
    for kind, pad in (("float32", None), ("bfloat16", 0), ("float16", None)):
        tokens = np.minimum((V * rng.random(n) ** 2).astype(np.int64), V - 1)
        dout = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).cuda().to(getattr(torch, kind))
        srv.emb_adagrad_step(torch.from_numpy(tokens).cuda(), dout, lr, eps, first_key=first, num_tokens=V, scale=0.7, pad_token=pad)
        g, mag, count = _sums(tokens, dout.double().cpu().numpy(), V, pad)
        s = np.float64(np.float32(0.7))
        g, mag = g * s, mag * s
        rows = slice(first, first + V)
        dg = mag * (64 + count / 8 + 3)[:, None] * 2.0 ** -24                      # what the sum may be off by
        hit = count > 0
        G = want[rows, D:2 * D] + g * g
        root = np.sqrt(G + np.float32(eps))
        err[rows, D:2 * D] += np.where(hit[:, None], 2 * np.abs(g) * dg + dg ** 2 + 4 * G * 2.0 ** -24, 0)
        # of lr g / root, |d/dg| <= lr / root, and of G through the root lr |g| / (2 root^3)
        err[rows, :D] += np.where(hit[:, None], np.float32(lr) * (dg / root + np.abs(g) * err[rows, D:2 * D] / (2 * root ** 3) + 8 * 2.0 ** -24 * (np.abs(g) / root))
                                  + 2.0 ** -23 * (np.abs(want[rows, :D]) + lr), 0)
        want[rows, :D] -= np.float32(lr) * g / root
        want[rows, D:2 * D] = G
    got = _all(srv)
    off = np.abs(got - want)
    assert (off <= err + 1e-12).all(), float((off - err).max())
    srv.status()
    srv2.status()


@pytest.mark.parametrize("n", [1, 300, 3000])
@pytest.mark.parametrize("caches", [0, 1])
def test_statistics_are_those_of_pull_and_push(n, caches):
    """A lookup is counted as a pull of the tokens' keys without the padding, a step as a pull and a push."""
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(n)
    K, L, W, first, V = 900, 16, 5, 100, 640
    a, b = P.ParameterServer(K, L, W), P.ParameterServer(K, L, W)
    for s in (a, b):
        s.set_option(P.OPT_LOCATION_CACHES, caches)
        s.localize(torch.arange(0, K, 3, device="cuda"), 2)
    for i in range(4):
        tokens = rng.integers(0, V, size=n)
        tokens[rng.random(n) < 0.2] = 17
        worker = int(rng.integers(-1, W))
        t, keys = torch.from_numpy(tokens.astype(np.int32 if i % 2 else np.int64)).cuda(), torch.from_numpy(tokens[tokens != 17] + first).cuda()
        a.emb_lookup(t, first_key=first, num_tokens=V, pad_token=17, worker=worker)
        b.pull(keys, worker)
        assert a.stats() == b.stats()
        a.emb_adagrad_step(t, torch.ones(n, 8, device="cuda"), 0.1, 1e-8, first_key=first, num_tokens=V, pad_token=17, worker=worker)
        b.pull(keys, worker)
        b.push(keys, torch.zeros(keys.numel(), L, device="cuda"), worker)
        assert a.stats() == b.stats()
        for s in (a, b):
            s.localize(torch.from_numpy(rng.integers(0, K, size=50)).cuda(), int(rng.integers(0, W))) if i < 0 else None
    assert torch.equal(a.owner(), b.owner())


@pytest.mark.parametrize("n", [1, 64, 2048, 2049, 140_000])
@pytest.mark.parametrize("bad", [-1, 640, 1 << 40])
def test_a_bad_token_changes_nothing(n, bad):
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(n)
    print(f"case n={n} bad={bad}", flush=True)
    srv, values = _server(900, 16, W=3)
    tokens = rng.integers(0, 640, size=n)
    tokens[int(rng.integers(0, n))] = bad
    t = torch.from_numpy(tokens).cuda()
    out, grad, dout = torch.full((n, 16), 7.0, device="cuda"), torch.full((640, 8), 7.0, device="cuda"), torch.ones(n, 8, device="cuda")
    stats = srv.stats()
    for call in (lambda: srv.emb_lookup(t, num_tokens=640, out=out, worker=1), lambda: srv.emb_grad(t, dout, 640, grad=grad),
                 lambda: srv.emb_grad(t, dout, 640, grad=grad, accumulate=True),
                 lambda: srv.emb_adagrad_step(t, dout, 0.1, 1e-8, num_tokens=640, worker=1)):
        call()
        call()                                                    # (nor does a later call before the status is asked for)
        with pytest.raises(P.PSError) as e:
            srv.status()
        assert e.value.code == P.PS_EKEY
    assert (out == 7.0).all() and (grad == 7.0).all() and np.array_equal(_all(srv), values) and srv.stats() == stats
    # a pad token outside the vocabulary is no error
    srv.emb_lookup(t, num_tokens=640, pad_token=bad)
    srv.status()


@pytest.mark.parametrize("n", [1, 64, 2048, 2049, 5000, 10_000, 140_000])
def test_the_lowest_token_is_a_bad_one_where_there_is_no_padding(n):
    """PS_NO_PAD has a value that an int64 batch can hold: an error like any other token that is not there."""
    import torch
    from paper_2002_00655_amd import ps as P
    rng = np.random.default_rng(n)
    srv, values = _server(900, 16, W=3)
    tokens = rng.integers(0, 640, size=n)
    tokens[n // 2] = -(1 << 63)
    t = torch.from_numpy(tokens).cuda()
    out, grad, dout = torch.full((n, 16), 7.0, device="cuda"), torch.full((640, 8), 7.0, device="cuda"), torch.ones(n, 8, device="cuda")
    stats = srv.stats()
    for call in (lambda: srv.emb_lookup(t, num_tokens=640, out=out, worker=1), lambda: srv.emb_grad(t, dout, 640, grad=grad),
                 lambda: srv.emb_grad(t, dout, 640, grad=grad, accumulate=True),
                 lambda: srv.emb_adagrad_step(t, dout, 0.1, 1e-8, num_tokens=640, worker=1), lambda: srv.emb_lookup(t, num_tokens=640, out=out, pad_token=0),
                 lambda: srv.emb_grad(t, dout, 640, grad=grad, pad_token=-1)):
        call()
        with pytest.raises(P.PSError) as e:
            srv.status()
        assert e.value.code == P.PS_EKEY
    assert (out == 7.0).all() and (grad == 7.0).all() and np.array_equal(_all(srv), values) and srv.stats() == stats


def test_refusals():
    import torch
    from paper_2002_00655_amd import ps as P
    srv, values = _server(100, 16, W=2)
    t, dout = torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda")
    bad = [(P.PS_EINVAL, lambda: srv.emb_lookup(t, dim=17)), (P.PS_EINVAL, lambda: srv.emb_lookup(t, first_key=50, num_tokens=51)),
           (P.PS_EINVAL, lambda: srv.emb_lookup(t, first_key=-1, num_tokens=5)), (P.PS_EINVAL, lambda: srv.emb_lookup(t, num_tokens=0)),
           (P.PS_EWORKER, lambda: srv.emb_lookup(t, worker=2)), (P.PS_EWORKER, lambda: srv.emb_lookup(t, worker=-2)),
           (P.PS_EINVAL, lambda: srv.emb_adagrad_step(t, torch.zeros(5, 9, device="cuda"), 0.1, 1e-8)),
           (P.PS_EINVAL, lambda: srv.emb_adagrad_step(t, dout, 0.1, 0.0)), (P.PS_EINVAL, lambda: srv.emb_adagrad_step(t, dout, 0.1, float("nan"))),
           (P.PS_EWORKER, lambda: srv.emb_adagrad_step(t, dout, 0.1, 1e-8, worker=2)), (P.PS_EINVAL, lambda: srv.emb_adagrad_step(t, dout, 0.1, 1e-8, first_key=100)),
           (P.PS_EINVAL, lambda: srv.emb_grad(t, dout, 0))]
    for code, call in bad:
        with pytest.raises(P.PSError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: srv.emb_lookup(t.float()), lambda: srv.emb_lookup(t.cpu()), lambda: srv.emb_lookup(t, dtype=torch.float64), lambda: srv.emb_grad(t, dout.double(), 5),
                 lambda: srv.emb_grad(t, dout, 5, grad=torch.zeros(5, 8, device="cuda", dtype=torch.float16))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: srv.emb_grad(t, dout[:4], 5), lambda: srv.emb_grad(t, dout, 5, accumulate=True), lambda: srv.emb_lookup(t, out=torch.zeros(5, 15, device="cuda")),
                 lambda: srv.emb_grad(t, dout, 5, grad=torch.zeros(6, 8, device="cuda")), lambda: srv.emb_grad(t, torch.zeros(8, 5, device="cuda").t(), 5),
                 lambda: srv.emb_lookup(t.view(5, 1), out=torch.zeros(1, 5, 16, device="cuda").transpose(0, 1)[:, :, ::1][:, :, :15])):
        with pytest.raises(ValueError):
            call()
    srv.status()
    assert np.array_equal(_all(srv), values)


def test_calls_on_another_stream_and_in_a_graph():
    """The calls go to the current stream; once scratch has its size they can be captured, and replays see new inputs."""
    import torch
    rng = np.random.default_rng(3)
    V, D, n = 500, 64, 3000
    srv, _ = _server(V, 2 * D)
    ref, _ = _server(V, 2 * D)
    t = torch.from_numpy(rng.integers(0, V, size=n)).cuda()
    dout, out, grad = torch.zeros(n, D, device="cuda"), torch.zeros(n, D, device="cuda", dtype=torch.bfloat16), torch.zeros(V, D, device="cuda")

    def step(s):
        s.emb_lookup(t, dim=D, scale=2.0, out=out)
        s.emb_grad(t, dout, V, grad=grad)
        s.emb_adagrad_step(t, dout, 0.1, 1e-8)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(srv)
    torch.cuda.current_stream().wait_stream(side)
    step(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(srv)
    for i in range(3):
        t.copy_(torch.from_numpy(rng.integers(0, V, size=n)))
        dout.copy_(torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        a = out.clone(), grad.clone()
        step(ref)
        assert torch.equal(a[0], out) and torch.equal(a[1], grad) and np.array_equal(_all(srv), _all(ref)), i
