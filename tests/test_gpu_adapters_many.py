"""So many adapters that their matrices are not laid any more; numbers of 0 and 1, whose products and sums are exact in fp16."""
import pytest

pytestmark = pytest.mark.gpu


def test_thousands_of_adapters():
    import torch
    from paper_2002_00655_amd import ps as P
    adapters, rank, rows, dim, each = 17000, 4, 1024, 64, 64
    n, W = adapters * each, adapters * rank
    g = torch.Generator(device="cuda").manual_seed(1)
    values = torch.randint(0, 2, (rows + 2 * W, 1024), device="cuda", generator=g, dtype=torch.int8).float()
    srv = P.ParameterServer(values.shape[0], 1024, 1)
    srv.push(torch.arange(values.shape[0], device="cuda"), values)
    w, a, b = values[:rows, :dim].contiguous(), values[rows:rows + W, :dim].reshape(adapters, rank, dim), values[rows + W:].view(adapters, rank, rows)
    place = torch.randperm(n, device="cuda", generator=g)                    # row place[i] has adapter i / each
    ids = torch.empty(n, dtype=torch.int32, device="cuda")
    ids[place] = (torch.arange(n, device="cuda") // each).int()
    groups = srv.group_rows(ids, adapters)
    x = torch.randint(0, 2, (n, dim), device="cuda", generator=g, dtype=torch.int8).half()
    dout = torch.zeros(n, rows, dtype=torch.float16, device="cuda")
    dout[:, ::64] = torch.randint(0, 2, (n, rows // 64), device="cuda", generator=g, dtype=torch.int8).half()
    print("forward", flush=True)
    out = srv.adapter_matmul(x, groups, 0, rows, rows, rows + W, rank, dim=dim)
    print("gradient", flush=True)
    dx, da, db = srv.adapter_grad(x, dout, groups, 0, rows, rows + W, rank)
    srv.status()
    for e0 in range(0, adapters, 1000):
        p = place[e0 * each:(e0 + 1000) * each]
        xs, ds, ae, be = x[p].float().view(1000, each, dim), dout[p].float().view(1000, each, rows), a[e0:e0 + 1000].contiguous(), b[e0:e0 + 1000].contiguous()
        h, t = torch.bmm(xs, ae.transpose(1, 2).contiguous()), torch.bmm(ds, be.transpose(1, 2).contiguous())
        want = (xs.view(-1, dim) @ w.t().contiguous()).view(1000, each, rows) + torch.bmm(h, be)
        assert want.max() <= 2048 and torch.equal(out[p].float().view_as(want), want), e0
        want = (ds.view(-1, rows) @ w).view(1000, each, dim) + torch.bmm(t, ae)
        assert want.max() <= 2048 and torch.equal(dx[p].float().view_as(want), want), e0
        assert torch.equal(da[e0:e0 + 1000], torch.bmm(t.transpose(1, 2).contiguous(), xs)), e0
        assert torch.equal(db[e0:e0 + 1000], torch.bmm(h.transpose(1, 2).contiguous(), ds)), e0
