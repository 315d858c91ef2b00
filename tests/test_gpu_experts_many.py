"""A few rows of very many experts; numbers whose products are exact."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("experts,rows,dim", [(65536, 4096, 1), (65536, 300, 3), (5000, 65, 24)])
def test_few_rows_of_many_experts(experts, rows, dim, kind):
    import torch
    from paper_2002_00655_amd import ps as P
    print("case", experts, rows, dim, kind, flush=True)
    srv = P.ParameterServer(experts * rows, dim, 1)
    keys = torch.arange(experts * rows, device="cuda")
    for i in range(0, experts * rows, 1 << 24):                              # number c of key k: (k + c) mod 127
        k = keys[i:i + (1 << 24)]
        srv.push(k, ((k[:, None] + torch.arange(dim, device="cuda")) % 127).float())
    for chosen in ([experts - 1], [0, experts - 1, -1, experts // 2, 0], list(range(experts - 40, experts))):
        n = len(chosen)
        ids = torch.tensor(chosen, device="cuda")
        groups = srv.group_rows(ids, experts, pad=-1)
        w = torch.stack([srv.pull(keys[max(e, 0) * rows:(max(e, 0) + 1) * rows]) * (e >= 0) for e in chosen])
        for transposed in (False, True):
            x = torch.zeros(n, rows if transposed else dim, device="cuda")
            x[:, ::max(1, x.shape[1] // 2)] = 1.0
            out = srv.expert_matmul(x.to(getattr(torch, kind)), groups, 0, rows, dim=dim, transposed=transposed, dtype=torch.float32)
            want = torch.bmm(w.transpose(1, 2).contiguous() if transposed else w, x[:, :, None])[:, :, 0]
            assert torch.equal(out, want), (chosen[:3], transposed)
    srv.status()


@pytest.mark.parametrize("n,dim,pairs", [(2 * ((1 << 20) + 3), 1024, 2), (3 * 90001, 13, 3)])
def test_sums_over_pairs_of_many_rows(n, dim, pairs):
    """More numbers than one round of the sums' workgroups takes."""
    import torch
    from paper_2002_00655_amd import ps as P
    experts, rows = 2, 8
    srv = P.ParameterServer(experts * rows, dim, 1)
    g = torch.Generator(device="cuda").manual_seed(n)
    w = torch.randint(0, 2, (experts * rows, dim), device="cuda", generator=g).float()
    srv.push(torch.arange(experts * rows, device="cuda"), w)
    ids = torch.randint(-1, experts, (n,), device="cuda", generator=g)
    x = torch.randint(0, 2, (n, rows), device="cuda", generator=g).bfloat16()
    out = srv.expert_matmul(x, srv.group_rows(ids, experts, pad=-1), 0, rows, transposed=True, sum_pairs=pairs)
    for i in range(0, n, 300 * 1000 * pairs):
        j = min(n, i + 300 * 1000 * pairs)
        want = sum((x[i:j].float() * (ids[i:j] == e)[:, None]) @ w[e * rows:(e + 1) * rows] for e in range(experts))
        assert torch.equal(out[i // pairs:j // pairs].float(), want.view(-1, pairs, dim).sum(1)), i
    srv.status()
