"""What the operators of token models on the server are measured on: a lookup of token embeddings, its gradient, a step
of AdaGrad on the looked-up rows, and the orthogonalised update of weight matrices.

Five kinds of pass:

``lookup``   the scaled embeddings of a batch of tokens, in the type that the model computes in;
``grad``     the gradient of such a lookup with respect to the whole table, from the gradient of its output;
``adagrad``  a step of AdaGrad on the rows that a batch mentions, the accumulators next to the values, and the rows of
             the batch read back, as the next step of the program does;
``orth``     matrices (momenta, updates) orthogonalised by Newton-Schulz products;
``muon``     a step of a weight matrix that lies in the server, its momentum next to it, and the matrix read back.

Where ``own`` is false a pass is the operator written down in elementary torch operations in 32 bits; where it is true it
is the call of ``paper_2002_00655_amd.ps`` that a user makes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
LR, EPS = 0.05, 1e-8                                # AdaGrad
MU, MUON_LR, DECAY = 0.95, 0.02, 0.01               # the orthogonalised update
STEPS, NORM_EPS = 5, 1e-7
A, B, C = 3.4445, -4.7750, 2.0315
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOKENS = {"i32": torch.int32, "i64": torch.int64}


# ---- the cases ----------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of a sequence that is being generated: what a call costs
        dict(name="lookup_one", kind="lookup", n=1, vocab=32_000, dim=512, length=512, tokens="i32", type="bf16", pad=False, skew=0.0),
        # a training batch of long sequences, some of them padded, the accumulators lying between the rows
        dict(name="lookup_batch", kind="lookup", n=65_537, vocab=50_000, dim=512, length=1024, tokens="i64", type="bf16", pad=True, skew=1.0),
        # a small table (positions, types of a token; here entities of a small graph) and few tokens, rows of 100
        dict(name="grad_small", kind="grad", n=333, vocab=5000, dim=100, tokens="i32", type="f32", pad=False, skew=1.0, add=False),
        # one sequence of ordinary length: the table is larger than what is added to it
        dict(name="grad_sequence", kind="grad", n=16_384, vocab=50_000, dim=1024, tokens="i64", type="bf16", pad=True, skew=1.0, add=False),
        # a large batch onto the gradient of the batches before it, frequent tokens ten thousands of times
        dict(name="grad_batch", kind="grad", n=262_144, vocab=128_000, dim=512, tokens="i32", type="bf16", pad=False, skew=1.0, add=True),
        # the tokens of a few data points
        dict(name="adagrad_few", kind="adagrad", n=64, vocab=20_001, dim=128, tokens="i32", type="f32", pad=False, skew=1.0),
        # a training batch
        dict(name="adagrad_batch", kind="adagrad", n=65_536, vocab=100_000, dim=512, tokens="i64", type="bf16", pad=True, skew=1.0),
        # many small matrices, of the rank of the factorization benchmarks
        dict(name="orth_many_small", kind="orth", batch=16, rows=100, cols=100, type="f32"),
        # a projection of a wide layer, in 32 bits
        dict(name="orth_tall", kind="orth", batch=1, rows=4096, cols=1024, type="f32"),
        # the largest: square, in 16 bits
        dict(name="orth_square", kind="orth", batch=2, rows=4096, cols=4096, type="bf16"),
        # one matrix of a small model, sides that are no multiple of anything
        dict(name="muon_small", kind="muon", batch=1, rows=333, dim=127, type="f32"),
        # the matrices of eight layers
        dict(name="muon_layers", kind="muon", batch=8, rows=2048, dim=512, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "grad", "adagrad", "orth", "muon"])
    kinds = rng.choice(["i32", "i64"]), rng.choice(["f32", "bf16", "f16"])
    dims = [16, 50, 64, 100, 128, 400, 512, rng.randint(1, 512)]
    if kind == "lookup":
        length = rng.choice(dims + [1024, rng.randint(512, 1024)])
        dim = rng.choice([length, length, (length + 1) // 2])
        return dict(kind=kind, n=_log_int(rng, 1, 65_536), vocab=_log_int(rng, 500, 100_000), dim=dim, length=length, tokens=kinds[0], type=kinds[1],
                    pad=rng.random() < 0.3, skew=rng.choice([0.0, 1.0]))
    if kind == "grad":
        dim = rng.choice(dims + [1024, rng.randint(512, 1024)])
        n, vocab = min(_log_int(rng, 1, 262_144), 262_144 * 256 // dim), min(_log_int(rng, 100, 128_000), 128_000 * 512 // dim)
        return dict(kind=kind, n=n, vocab=vocab, dim=dim, tokens=kinds[0], type=kinds[1], pad=rng.random() < 0.3, skew=rng.choice([0.0, 1.0, 1.2]), add=rng.random() < 0.3)
    if kind == "adagrad":
        return dict(kind=kind, n=_log_int(rng, 1, 65_536), vocab=_log_int(rng, 100, 100_000), dim=rng.choice(dims), tokens=kinds[0], type=kinds[1],
                    pad=rng.random() < 0.3, skew=rng.choice([0.0, 1.0, 1.2]))
    if kind == "orth":
        rows, cols = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        batch = max(1, min(_log_int(rng, 1, 64), (1 << 24) // (rows * cols)))
        return dict(kind=kind, batch=batch, rows=rows, cols=cols, type=rng.choice(["f32", "bf16"]))
    rows, dim = _log_int(rng, 1, 4096), rng.choice([64, 128, 256, 512, _log_int(rng, 1, 512)])
    return dict(kind=kind, batch=max(1, min(_log_int(rng, 1, 32), (1 << 23) // (rows * dim))), rows=rows, dim=dim, type=kinds[1])


# ---- inputs -------------------------------------------------------------------------------------------------------
def _probs(c):
    """How often the frequent tokens come: rank^-skew."""
    p = np.arange(1, c["vocab"] + 1, dtype=np.float64) ** -c["skew"]
    return p / p.sum()


def _tokens(c, g):
    """Token ids, frequent ones anywhere in the table; of a padded batch about an eighth is padding, at its end."""
    cdf = torch.from_numpy(np.cumsum(_probs(c))).to(DEV)
    u = torch.rand(c["n"], device=DEV, generator=g, dtype=torch.float64)
    ids = torch.searchsorted(cdf, u, right=True).clamp_(max=c["vocab"] - 1)
    ids = torch.randperm(c["vocab"], device=DEV, generator=g)[ids]
    if c["pad"]:
        ids[c["n"] - (c["n"] + 4) // 8:] = _pad(c)
    return ids.to(TOKENS[c["tokens"]])


def _pad(c):
    return 0 if c["pad"] else None


def _matrices(c, g, cols):
    """Gradients of weight matrices: a few strong directions and, under them, noise in all others."""
    r = max(1, min(8, c["rows"], cols) // 2)
    u = torch.randn(c["batch"], c["rows"], r, device=DEV, generator=g)
    v = torch.randn(c["batch"], r, cols, device=DEV, generator=g)
    x = torch.matmul(u, v) * (1.0 / math.sqrt(r)) + torch.randn(c["batch"], c["rows"], cols, device=DEV, generator=g)
    return (x * 1e-3).to(TYPES[c["type"]])


def _server(values):
    """A server that holds these rows."""
    from paper_2002_00655_amd import ps as P
    srv = P.ParameterServer(values.shape[0], values.shape[1], 1)
    srv.push(torch.arange(values.shape[0], device=DEV), values)
    return srv


def _handle():
    from paper_2002_00655_amd import ps as P
    return P.ParameterServer(1, 1, 1)


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case=c)
    if c["kind"] == "orth":
        s["x"] = _matrices(c, g, c["cols"])
        if own:
            s["server"] = _handle()
        return s
    if c["kind"] == "muon":
        rows = c["batch"] * c["rows"]
        s["grad"] = _matrices(c, g, c["dim"])
        weight = torch.randn(rows, c["dim"], device=DEV, generator=g) * 0.02
        moment = torch.randn(rows, c["dim"], device=DEV, generator=g) * 4e-3
        s["keys"], values = torch.arange(rows, device=DEV), torch.cat([weight, moment], 1)
        s["server" if own else "values"] = _server(values) if own else values
        return s
    s["tokens"] = _tokens(c, g)
    if c["kind"] == "lookup":
        values = torch.randn(c["vocab"], c["length"], device=DEV, generator=g) * 0.02
        s["server" if own else "values"] = _server(values) if own else values
        return s
    s["dout"] = (torch.randn(c["n"], c["dim"], device=DEV, generator=g) * 0.01).to(TYPES[c["type"]])
    if c["kind"] == "grad":
        s["grad"] = torch.randn(c["vocab"], c["dim"], device=DEV, generator=g) * 0.01 if c["add"] else torch.empty(c["vocab"], c["dim"], device=DEV)
        if own:
            s["server"] = _handle()
        return s
    s["keys"] = s["tokens"].long()
    values = torch.cat([torch.randn(c["vocab"], c["dim"], device=DEV, generator=g) * 0.02, torch.rand(c["vocab"], c["dim"], device=DEV, generator=g) * 1e-3], 1)
    s["server" if own else "values"] = _server(values) if own else values
    return s


# ---- a pass -------------------------------------------------------------------------------------------------------
def run(state):
    return (run_own if own else run_plain)[state["case"]["kind"]](state, state["case"])


def _scale(c):
    return math.sqrt(c["dim"])


def _terms(s, c):
    """The scaled rows of the output's gradient, those of padding zero."""
    rows = s["dout"].float() * _scale(c)
    if c["pad"]:
        rows = torch.where((s["tokens"] == _pad(c))[:, None], torch.zeros((), device=DEV), rows)
    return rows


def _plain_lookup(s, c):
    tokens = s["tokens"].long()
    out = s["values"][tokens, :c["dim"]] * _scale(c)
    if c["pad"]:
        out = torch.where((tokens == _pad(c))[:, None], torch.zeros((), device=DEV), out)
    return out.to(TYPES[c["type"]])


def _plain_grad(s, c):
    into = s["grad"] if c["add"] else torch.zeros(c["vocab"], c["dim"], device=DEV)
    return into.index_add_(0, s["tokens"].long(), _terms(s, c))


def _plain_adagrad(s, c):
    # (padding has a gradient of zero, and a row with a gradient of zero stays as it is)
    d, values = c["dim"], s["values"]
    keys, place = torch.unique(s["tokens"].long(), return_inverse=True)
    g = torch.zeros(keys.numel(), d, device=DEV).index_add_(0, place, _terms(s, c))
    rows = values[keys]
    acc = rows[:, d:] + g * g
    values[keys] = torch.cat([rows[:, :d] - LR * g / torch.sqrt(acc + EPS), acc], 1)
    return values[s["keys"]]


def _newton_schulz(x):
    """[batch, rows, cols] in 32 bits."""
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + NORM_EPS)
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.matmul(B * gram + C * torch.matmul(gram, gram), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_orth(s, c):
    return _newton_schulz(s["x"].float()).to(TYPES[c["type"]])


def _plain_muon(s, c):
    d, g, values = c["dim"], s["grad"].float(), s["values"]
    rows = values[s["keys"]].view(c["batch"], c["rows"], 2 * d)
    moment = MU * rows[:, :, d:] + g
    o = _newton_schulz(g + MU * moment)
    weight = (1 - MUON_LR * DECAY) * rows[:, :, :d] - MUON_LR * math.sqrt(max(1.0, c["rows"] / d)) * o
    values[s["keys"]] = torch.cat([weight, moment], 2).view(-1, 2 * d)
    return values[s["keys"]]


run_plain = dict(lookup=_plain_lookup, grad=_plain_grad, adagrad=_plain_adagrad, orth=_plain_orth, muon=_plain_muon)


def _own_lookup(s, c):
    return s["server"].emb_lookup(s["tokens"], dim=c["dim"], scale=_scale(c), pad_token=_pad(c), dtype=TYPES[c["type"]])


def _own_grad(s, c):
    return s["server"].emb_grad(s["tokens"], s["dout"], c["vocab"], scale=_scale(c), pad_token=_pad(c), grad=s["grad"] if c["add"] else None, accumulate=c["add"])


def _own_adagrad(s, c):
    s["server"].emb_adagrad_step(s["tokens"], s["dout"], LR, EPS, scale=_scale(c), pad_token=_pad(c))
    return s["server"].pull(s["keys"])


def _own_orth(s, c):
    return s["server"].muon_orthogonalize(s["x"], steps=STEPS, eps=NORM_EPS)


def _own_muon(s, c):
    s["server"].muon_step(0, s["grad"], MUON_LR, momentum=MU, nesterov=True, weight_decay=DECAY, steps=STEPS, eps=NORM_EPS)
    return s["server"].pull(s["keys"])


run_own = dict(lookup=_own_lookup, grad=_own_grad, adagrad=_own_adagrad, orth=_own_orth, muon=_own_muon)


# ---- the result in 64 bits ----------------------------------------------------------------------------------------
def _exact_sums(tokens, dout, c):
    """The distinct tokens (without padding) in order and their sums: differences of running sums over the sorted rows."""
    keep = tokens != _pad(c) if c["pad"] else torch.ones_like(tokens, dtype=torch.bool)
    ids, order = torch.sort(tokens[keep].long(), stable=True)
    keys, counts = torch.unique_consecutive(ids, return_counts=True)
    ends = torch.cumsum(counts, 0)
    rows, parts = dout[keep][order], []
    for c0 in range(0, c["dim"], 128):
        total = torch.cumsum(rows[:, c0:c0 + 128].double() * math.sqrt(c["dim"]), 0)
        total = torch.cat([torch.zeros(1, total.shape[1], dtype=torch.float64, device=DEV), total])[torch.cat([ends.new_zeros(1), ends])]
        parts.append(total[1:] - total[:-1])
    return keys, torch.cat(parts, 1)


def _exact_orth(x):
    """By the shorter side's Gram matrix on the right: x p(x'x), in 64 bits."""
    x = x.double()
    if x.shape[1] < x.shape[2]:
        return _exact_orth(x.transpose(1, 2)).transpose(1, 2)
    out = torch.empty_like(x)
    for i in range(x.shape[0]):
        y = x[i].contiguous()
        y = y / (torch.linalg.vector_norm(y) + NORM_EPS)
        for _ in range(STEPS):
            h = torch.mm(y.t().contiguous(), y)
            y = torch.addmm(y, y, torch.addmm(h, h, h, beta=B, alpha=C), beta=A)
        out[i] = y
    return out


def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    if c["kind"] == "lookup":
        out = s["values"].double()[s["tokens"].long(), :c["dim"]] * math.sqrt(c["dim"])
        if c["pad"]:
            out[s["tokens"] == _pad(c)] = 0.0
        return out
    if c["kind"] == "grad":
        keys, sums = _exact_sums(s["tokens"], s["dout"], c)
        out = s["grad"].double() if c["add"] else torch.zeros(c["vocab"], c["dim"], dtype=torch.float64, device=DEV)
        out[keys] += sums
        return out
    if c["kind"] == "adagrad":
        d, values = c["dim"], s["values"].double()
        keys, g = _exact_sums(s["tokens"], s["dout"], c)
        values[keys, d:] += g ** 2
        values[keys, :d] -= LR * g * (values[keys, d:] + EPS) ** -0.5
        return values[s["keys"]]
    if c["kind"] == "orth":
        return _exact_orth(s["x"])
    d, g, values = c["dim"], s["grad"].double(), s["values"].double().view(c["batch"], c["rows"], -1)
    moment = values[:, :, d:] * MU + g
    weight = values[:, :, :d] * (1 - MUON_LR * DECAY) - _exact_orth(g + moment * MU) * (MUON_LR * max(1.0, c["rows"] / d) ** 0.5)
    return torch.cat([weight, moment], 2).view(-1, 2 * d)


# ---- the work -----------------------------------------------------------------------------------------------------
def work(case):
    c = case
    size = 4 if c["type"] == "f32" else 2
    if c["kind"] in ("orth", "muon"):
        cols = c["cols"] if c["kind"] == "orth" else c["dim"]
        n, m = min(c["rows"], cols), max(c["rows"], cols)
        # the Gram matrix and its square are symmetric: half of their products
        flops = STEPS * c["batch"] * (n * n * m + n ** 3 + 2 * n * n * m)
        values = c["batch"] * n * m
        # the orthogonalised matrices; the step: the gradient, values and momentum in and out, both read back
        return dict(bytes=2.0 * size * values if c["kind"] == "orth" else (size + 16.0 + 16.0) * values, flops=float(flops))
    n = c["n"] - (c["n"] + 4) // 8 if c["pad"] else c["n"]
    rows = float((-np.expm1(n * np.log1p(-np.minimum(_probs(c), 1 - 1e-12)))).sum())          # distinct tokens to be expected
    ids = c["n"] * (4 if c["tokens"] == "i32" else 8)
    if c["kind"] == "lookup":
        return dict(bytes=ids + 4.0 * rows * c["dim"] + size * c["n"] * c["dim"], flops=float(n * c["dim"]))
    terms = ids + float(size) * n * c["dim"]
    if c["kind"] == "grad":
        return dict(bytes=terms + (8.0 * rows if c["add"] else 4.0 * c["vocab"]) * c["dim"], flops=2.0 * n * c["dim"])
    # values and accumulators in and out, both read back for every token
    return dict(bytes=terms + ((16.0 + 8.0) * rows + 8.0 * c["n"]) * c["dim"], flops=(2.0 * n + 7.0 * rows) * c["dim"])
