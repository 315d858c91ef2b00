"""What the operators of models with many matrices on the server are measured on: rows grouped by the matrix they use, products
with experts and their gradients, and products with a shared projection and a low-rank adapter per request.

Five kinds of pass:

``group``          the order of rows by group and where the groups start, from the rows' group ids;
``experts``        rows grouped by expert and multiplied by its matrix, or (``down``) by its transpose and added up per token;
``experts_back``   the gradients of such a product: of its rows and of all matrices;
``adapters``       rows grouped by adapter and multiplied by a shared matrix and, beside it, by their adapter's two;
``adapters_back``  the gradients of that: of the rows and of all adapters.

Where ``own`` is false a pass is the operator written down in elementary torch operations in 32 bits; where it is true it
is the calls of ``paper_2002_00655_amd.ps`` that a user makes.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IDS = {"i32": torch.int32, "i64": torch.int64}
PAD = -1
MOST = 1.4e11                                       # operations of a drawn case


# ---- the cases ----------------------------------------------------------------------------------------------------
def listed():
    return [
        # the experts of a few sequences' next tokens
        dict(name="group_few", kind="group", n=128, groups=16, ids="i64", pad=False, skew=0.0),
        # a large training batch, tokens beyond an expert's capacity dropped
        dict(name="group_batch", kind="group", n=131_072, groups=64, ids="i32", pad=True, skew=1.0),
        # one token of a sequence that is being generated, two experts of eight
        dict(name="experts_one", kind="experts", down=False, tokens=1, k=2, experts=8, rows=512, dim=512, length=512, type="bf16", pad=False, skew=0.0),
        # the next tokens of 64 sequences, the optimiser's momentum lying between the rows
        dict(name="experts_decode", kind="experts", down=False, tokens=64, k=2, experts=16, rows=1024, dim=512, length=1024, type="f16", pad=False, skew=0.5),
        # a small model in 32 bits, sides that are no multiple of anything, back to the model's width
        dict(name="experts_down", kind="experts", down=True, tokens=1999, k=2, experts=7, rows=400, dim=127, length=254, type="f32", pad=True, skew=0.5),
        # the largest: a training batch, some experts asked for much more than others
        dict(name="experts_batch", kind="experts", down=False, tokens=16_384, k=2, experts=16, rows=2048, dim=1024, length=1024, type="bf16", pad=False, skew=0.7),
        # a small batch's gradients in 32 bits, at the rank of the factorization benchmarks
        dict(name="experts_back_small", kind="experts_back", tokens=333, k=1, experts=5, rows=400, dim=100, length=200, type="f32", pad=True, skew=0.5),
        # a training batch's gradients
        dict(name="experts_back_batch", kind="experts_back", tokens=8192, k=2, experts=8, rows=1024, dim=512, length=1024, type="bf16", pad=False, skew=0.7),
        # the next tokens of 64 requests, each with one of 200 adapters
        dict(name="adapters_decode", kind="adapters", n=64, requests=64, adapters=200, rank=16, rows=1024, dim=1024, length=1024, type="bf16", skew=0.5),
        # the prompts of 24 requests
        dict(name="adapters_prompts", kind="adapters", n=16_001, requests=24, adapters=64, rank=32, rows=1024, dim=1024, length=1024, type="bf16", skew=0.5),
        # sequences of a few adapters that are being trained, in 32 bits, sides of no multiple
        dict(name="adapters_back_small", kind="adapters_back", n=333, requests=9, adapters=6, rank=5, rows=100, dim=127, length=254, type="f32", skew=0.0),
        # a batch of 32 sequences onto 16 adapters
        dict(name="adapters_back_batch", kind="adapters_back", n=16_384, requests=32, adapters=16, rank=16, rows=512, dim=512, length=1024, type="bf16", skew=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _side(rng, hi):
    return min(hi, rng.choice([64, 100, 128, 400, 512, 1024, _log_int(rng, 1, hi), _log_int(rng, 64, hi)]))


def draw(rng):
    kind = rng.choice(["group", "experts", "experts", "experts_back", "adapters", "adapters_back"])
    skew, pad, type_ = rng.choice([0.0, 0.5, 1.0]), rng.random() < 0.3, rng.choice(["f32", "bf16", "f16"])
    if kind == "group":
        return dict(kind=kind, n=_log_int(rng, 1, 131_072), groups=_log_int(rng, 1, 512), ids=rng.choice(["i32", "i64"]), pad=pad, skew=skew)
    dim = _side(rng, 1024)
    length = rng.choice([dim, min(1024, 2 * dim), 1024])
    if kind in ("experts", "experts_back"):
        experts, rows = _log_int(rng, 1, 64), _side(rng, 2048)
        most = MOST / (2.0 * rows * dim * (2 if kind == "experts_back" else 1))
        pairs = min(_log_int(rng, 1, 32_768), max(1, int(most)))
        k = min(rng.choice([1, 1, 2, 4]), experts, pairs)
        c = dict(kind=kind, tokens=max(1, pairs // k), k=k, experts=experts, rows=rows, dim=dim, length=length, type=type_, pad=pad, skew=skew)
        if kind == "experts":
            c["down"] = rng.random() < 0.4
        return c
    rows, rank = _side(rng, 1024), rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)])
    n = _log_int(rng, 1, 16_384)
    return dict(kind=kind, n=n, requests=min(n, _log_int(rng, 1, 256)), adapters=_log_int(rng, 1, 256), rank=rank, rows=rows, dim=dim, length=max(length, rows), type=type_, skew=skew)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _shares(groups, skew):
    """How often groups are asked for: rank^-skew."""
    p = torch.arange(1, groups + 1, dtype=torch.float64) ** -skew
    return p / p.sum()


def _choices(rows, k, groups, skew, g):
    """k different groups for every row, the frequent ones anywhere."""
    p = _shares(groups, skew)[torch.randperm(groups, generator=torch.Generator().manual_seed(int(g.initial_seed())))].to(DEV)
    u = torch.rand(rows, groups, device=DEV, generator=g, dtype=torch.float64).clamp_(min=1e-300)
    return torch.topk(p.log() - torch.log(-torch.log(u)), k, dim=1).indices


def _dropped(ids, pad, g):
    if pad:
        ids = torch.where(torch.rand(ids.shape, device=DEV, generator=g) < 0.1, torch.full_like(ids, PAD), ids)
    return ids


def _pairs(c):
    return c["tokens"] * c["k"]


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _held(s, values):
    """The values in a server, or as they are."""
    if own:
        from paper_2002_00655_amd import ps as P
        s["server"] = P.ParameterServer(values.shape[0], values.shape[1], 1)
        s["server"].push(torch.arange(values.shape[0], device=DEV), values)
    else:
        s["values"] = values


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = dict(case=c)
    if c["kind"] == "group":
        s["ids"] = _dropped(_choices(c["n"], 1, c["groups"], c["skew"], g)[:, 0], c["pad"], g).to(IDS[c["ids"]])
        _held(s, torch.zeros(1, 1, device=DEV))
        return s
    values = 0.02 * _randn(g, _keys(c), c["length"])
    if c["kind"] in ("experts", "experts_back"):
        s["ids"] = _dropped(_choices(c["tokens"], c["k"], c["experts"], c["skew"], g), c["pad"], g).int()
        down = c["kind"] == "experts" and c["down"]
        s["x"] = _randn(g, _pairs(c) if down else c["tokens"], c["rows"] if down else c["dim"]).to(TYPES[c["type"]])
        if c["kind"] == "experts_back":
            s["dout"] = (0.01 * _randn(g, _pairs(c), c["rows"])).to(TYPES[c["type"]])
    else:
        # the rows of a request lie together; one request in eight has no adapter
        cuts = torch.sort(torch.randperm(c["n"] - 1, device=DEV, generator=g)[:c["requests"] - 1]).values + 1 if c["n"] > 1 else torch.zeros(0, device=DEV, dtype=torch.int64)
        which = _choices(c["requests"], 1, c["adapters"], c["skew"], g)[:, 0]
        which = torch.where(torch.rand(c["requests"], device=DEV, generator=g) < 0.125, torch.full_like(which, PAD), which)
        s["ids"] = which[torch.searchsorted(cuts, torch.arange(c["n"], device=DEV), right=True)].int()
        s["x"] = _randn(g, c["n"], c["dim"]).to(TYPES[c["type"]])
        if c["kind"] == "adapters_back":
            s["dout"] = (0.01 * _randn(g, c["n"], c["rows"])).to(TYPES[c["type"]])
    _held(s, values)
    if c["kind"].endswith("_back"):                 # the forward pass has made the groups
        if own:
            s["plan"] = s["server"].group_rows(s["ids"], _groups(c), pad=PAD)
        elif "experts" in c:
            s["plan"] = _plan(s["ids"], _groups(c))
    return s


def _groups(c):
    return c["experts"] if "experts" in c else c["adapters"]


def _keys(c):
    return c["experts"] * c["rows"] if "experts" in c else c["rows"] + 2 * c["adapters"] * c["rank"]


def _first_a(c):
    return c["rows"]


def _first_b(c):
    return c["rows"] + c["adapters"] * c["rank"]


def _scale(c):
    return 16.0 / c["rank"]


# ---- a pass -------------------------------------------------------------------------------------------------------
def run(state):
    return (run_own if own else run_plain)[state["case"]["kind"]](state, state["case"])


def _order(ids, groups):
    ids = ids.flatten().long()
    key = torch.where(ids == PAD, torch.full_like(ids, groups), ids)
    order = torch.sort(key, stable=True).indices
    offsets = (key[None, :] < torch.arange(groups + 1, device=DEV)[:, None]).sum(1)
    return order, offsets


def _plan(ids, groups):
    """The rows of every group, and where they lie if every group has a matrix of as many rows as the largest one."""
    order, offsets = _order(ids, groups)
    at = offsets.tolist()
    most, kept = max(b - a for a, b in zip(at, at[1:])), order[:at[-1]]
    group = torch.searchsorted(offsets, torch.arange(kept.numel(), device=DEV), right=True) - 1
    place = group * most + torch.arange(kept.numel(), device=DEV) - offsets[group]
    return dict(order=kept, at=at, most=most, place=place)


def _padded(rows, plan, groups):
    out = torch.zeros(groups * plan["most"], rows.shape[1], device=DEV)
    out[plan["place"]] = rows
    return out.view(groups, plan["most"], -1)


def _even(plan, groups):
    """Whether matrices of as many rows as the largest group are not much more than the groups' rows: one product of all then, else one each."""
    return groups * plan["most"] <= 1.25 * plan["order"].numel() + 4096


def _products(x, plan, m):
    """The rows x, in the groups' order, times their group's matrix."""
    groups = m.shape[0]
    if _even(plan, groups):
        return torch.bmm(_padded(x, plan, groups), m.contiguous()).view(groups * plan["most"], -1)[plan["place"]]
    out, at = torch.empty(x.shape[0], m.shape[2], device=DEV), plan["at"]
    for e in range(groups):
        torch.mm(x[at[e]:at[e + 1]], m[e], out=out[at[e]:at[e + 1]])
    return out


def _outer(left, right, plan, groups):
    """Per group, the sum of its rows' products left_i right_j."""
    if _even(plan, groups):
        return torch.bmm(_padded(left, plan, groups).transpose(1, 2).contiguous(), _padded(right, plan, groups))
    at = plan["at"]
    return torch.stack([torch.mm(left[at[e]:at[e + 1]].t(), right[at[e]:at[e + 1]]) for e in range(groups)])


def _back_in_place(rows, plan, n):
    out = torch.zeros(n, rows.shape[1], device=DEV)
    out[plan["order"]] = rows
    return out


def _plain_group(s, c):
    order, offsets = _order(s["ids"], c["groups"])
    return order.int(), offsets.int()


def _matrices(s, c):
    return s["values"].view(c["experts"], c["rows"], -1)[:, :, :c["dim"]]


def _plain_experts(s, c):
    x, plan, w = s["x"].float(), _plan(s["ids"], c["experts"]), _matrices(s, c)
    if c["down"]:
        out = _back_in_place(_products(x[plan["order"]], plan, w), plan, _pairs(c))
        return out.view(c["tokens"], c["k"], c["dim"]).sum(1).to(TYPES[c["type"]])
    return _back_in_place(_products(x[plan["order"] // c["k"]], plan, w.transpose(1, 2)), plan, _pairs(c)).to(TYPES[c["type"]])


def _plain_experts_back(s, c):
    plan = s["plan"]
    x, dout = s["x"].float()[plan["order"] // c["k"]], s["dout"].float()[plan["order"]]
    dx = _back_in_place(_products(dout, plan, _matrices(s, c)), plan, _pairs(c))
    return dx.view(c["tokens"], c["k"], c["dim"]).sum(1).to(TYPES[c["type"]]), _outer(dout, x, plan, c["experts"])


def _parts(s, c):
    """The shared matrix, and all adapters' rows A and B' below one another."""
    return s["values"][:c["rows"], :c["dim"]], s["values"][_first_a(c):_first_b(c), :c["dim"]], s["values"][_first_b(c):, :c["rows"]]


def _of_own(rows, s, c):
    """Rows times all adapters' rows, scaled; zero where the adapter is another row's."""
    which = torch.arange(c["adapters"], device=DEV).repeat_interleave(c["rank"])
    return torch.where(s["ids"][:, None] == which[None, :], _scale(c) * rows, torch.zeros((), device=DEV))


def _plain_adapters(s, c):
    x, (w, a, b) = s["x"].float(), _parts(s, c)
    return (torch.mm(x, w.t()) + torch.mm(_of_own(torch.mm(x, a.t()), s, c), b)).to(TYPES[c["type"]])


def _plain_adapters_back(s, c):
    x, dout, (w, a, b) = s["x"].float(), s["dout"].float(), _parts(s, c)
    h, t = _of_own(torch.mm(x, a.t()), s, c), _of_own(torch.mm(dout, b.t()), s, c)
    dx = torch.mm(dout, w) + torch.mm(t, a)
    return dx.to(TYPES[c["type"]]), torch.mm(t.t(), x).view(c["adapters"], c["rank"], -1), torch.mm(h.t(), dout).view(c["adapters"], c["rank"], -1)


run_plain = dict(group=_plain_group, experts=_plain_experts, experts_back=_plain_experts_back, adapters=_plain_adapters, adapters_back=_plain_adapters_back)


def _own_group(s, c):
    return s["server"].group_rows(s["ids"], c["groups"], pad=PAD)


def _own_experts(s, c):
    groups = s["server"].group_rows(s["ids"], c["experts"], pad=PAD)
    return s["server"].expert_matmul(s["x"], groups, 0, c["rows"], dim=c["dim"], transposed=c["down"], sum_pairs=c["k"] if c["down"] else 1)


def _own_experts_back(s, c):
    dx = s["server"].expert_matmul(s["dout"], s["plan"], 0, c["rows"], dim=c["dim"], transposed=True, sum_pairs=c["k"])
    return dx, s["server"].expert_grad(s["dout"], s["x"], s["plan"])


def _own_adapters(s, c):
    groups = s["server"].group_rows(s["ids"], c["adapters"], pad=PAD)
    return s["server"].adapter_matmul(s["x"], groups, 0, c["rows"], _first_a(c), _first_b(c), c["rank"], scale=_scale(c), dim=c["dim"])


def _own_adapters_back(s, c):
    return s["server"].adapter_grad(s["x"], s["dout"], s["plan"], 0, _first_a(c), _first_b(c), c["rank"], scale=_scale(c))


run_own = dict(group=_own_group, experts=_own_experts, experts_back=_own_experts_back, adapters=_own_adapters, adapters_back=_own_adapters_back)


# ---- the result in 64 bits ----------------------------------------------------------------------------------------
def _exact_experts(s, c, ids, w):
    """Token by token's j-th choice: the tokens that chose an expert there."""
    x, down, k = s["x"].double(), c.get("down", False), c["k"]
    out = torch.zeros(c["tokens"], k, c["dim"] if down else c["rows"], dtype=torch.float64, device=DEV)
    for e in range(c["experts"]):
        m = w[e * c["rows"]:(e + 1) * c["rows"], :c["dim"]].double()
        t, j = torch.nonzero(ids == e, as_tuple=True)
        out[t, j] = torch.matmul(x[t * k + j], m) if down else torch.matmul(x[t], m.t().contiguous())
    return out.sum(1) if down else out.view(-1, c["rows"])


def _exact_experts_back(s, c, ids, w):
    x, d, k = s["x"].double(), s["dout"].double().view(c["tokens"], c["k"], -1), c["k"]
    dx = torch.zeros(c["tokens"], c["dim"], dtype=torch.float64, device=DEV)
    dw = torch.zeros(c["experts"], c["rows"], c["dim"], dtype=torch.float64, device=DEV)
    for e in range(c["experts"]):
        m = w[e * c["rows"]:(e + 1) * c["rows"], :c["dim"]].double()
        for j in range(k):
            t = torch.nonzero(ids[:, j] == e)[:, 0]
            dx[t] += torch.matmul(d[t, j], m)
            dw[e] += torch.matmul(d[t, j].t().contiguous(), x[t])
    return dx, dw


def _exact_adapters(s, c, ids, w):
    """A request's matrix as a whole: the shared one and its adapter's two multiplied."""
    x, shared = s["x"].double(), w[:c["rows"], :c["dim"]].double()
    a_all = w[_first_a(c):_first_b(c), :c["dim"]].double().view(-1, c["rank"], c["dim"])
    b_all = w[_first_b(c):, :c["rows"]].double().view(-1, c["rank"], c["rows"])
    out = torch.empty(c["n"], c["rows"], dtype=torch.float64, device=DEV)
    for a in torch.unique(ids).tolist():
        m = shared if a == PAD else shared + _scale(c) * torch.matmul(b_all[a].t().contiguous(), a_all[a])
        out[ids == a] = torch.matmul(x[ids == a], m.t().contiguous())
    return out


def _exact_adapters_back(s, c, ids, w):
    x, d, shared = s["x"].double(), s["dout"].double(), w[:c["rows"], :c["dim"]].double()
    a_all = w[_first_a(c):_first_b(c), :c["dim"]].double().view(-1, c["rank"], c["dim"])
    b_all = w[_first_b(c):, :c["rows"]].double().view(-1, c["rank"], c["rows"])
    dx, da, db = torch.empty_like(x), torch.zeros_like(a_all), torch.zeros_like(b_all)
    for a in torch.unique(ids).tolist():
        here = ids == a
        if a == PAD:
            dx[here] = torch.matmul(d[here], shared)
            continue
        # with the whole matrix' gradient G = d'x: of A  s B'G, of B' s (G A')'
        dx[here] = torch.matmul(d[here], shared + _scale(c) * torch.matmul(b_all[a].t().contiguous(), a_all[a]))
        whole = torch.matmul(d[here].t().contiguous(), x[here])
        da[a] = _scale(c) * torch.matmul(b_all[a], whole)
        db[a] = _scale(c) * torch.matmul(a_all[a], whole.t().contiguous())
    return dx, da, db


def exact(case, seed):
    global own
    c, was = case, own
    if c["kind"] == "group":
        return None
    own = False
    s = prepare(case, seed)
    own = was
    f = dict(experts=_exact_experts, experts_back=_exact_experts_back, adapters=_exact_adapters, adapters_back=_exact_adapters_back)[c["kind"]]
    return f(s, c, s["ids"].long(), s["values"])


# ---- the work -----------------------------------------------------------------------------------------------------
def _asked(shares, times, each=1):
    """Groups to be expected among `times` choices (of `each` different ones)."""
    return float((1.0 - (1.0 - (shares * each).clamp(max=1.0)) ** times).sum())


def work(case):
    c = case
    if c["kind"] == "group":
        return dict(bytes=c["n"] * ((4 if c["ids"] == "i32" else 8) + 4.0) + 4.0 * (c["groups"] + 1), flops=float(c["n"]))
    size = 4 if c["type"] == "f32" else 2
    if "experts" in c:
        kept = _pairs(c) * (0.9 if c["pad"] else 1.0)
        asked = _asked(_shares(c["experts"], c["skew"]), c["tokens"] * (0.9 if c["pad"] else 1.0), c["k"])
        weights, flops = 4.0 * asked * c["rows"] * c["dim"], 2.0 * kept * c["rows"] * c["dim"]
        few, many = size * c["tokens"] * c["dim"], size * _pairs(c) * c["rows"]
        if c["kind"] == "experts":
            return dict(bytes=weights + few + many + 4.0 * _pairs(c), flops=flops)
        return dict(bytes=weights + 2.0 * few + many + 4.0 * _pairs(c) + 4.0 * c["experts"] * c["rows"] * c["dim"], flops=2.0 * flops)
    asked = _asked(_shares(c["adapters"], c["skew"]), c["requests"] * 0.875)
    weights = 4.0 * (c["rows"] * c["dim"] + asked * c["rank"] * (c["rows"] + c["dim"]))
    low = 2.0 * c["n"] * 0.875 * c["rank"] * (c["rows"] + c["dim"])
    flops = 2.0 * c["n"] * c["rows"] * c["dim"]
    if c["kind"] == "adapters":
        return dict(bytes=weights + size * c["n"] * (c["rows"] + c["dim"]) + 4.0 * c["n"], flops=flops + low)
    grads = 4.0 * c["adapters"] * c["rank"] * (c["rows"] + c["dim"])
    return dict(bytes=weights + grads + size * c["n"] * (c["rows"] + 2 * c["dim"]) + 4.0 * c["n"], flops=flops + 2.5 * low)
