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
