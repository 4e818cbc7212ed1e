"""Tensors of more than 2^31 elements: what lies at their ends is found and kept where it belongs."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U, BF = 2.0 ** -24, torch.bfloat16


def rows_of(rows, c, seed):
    """[rows][c] bf16, zeros but for the first rows and the last ones; and where those are."""
    g = torch.Generator().manual_seed(seed)
    t = torch.zeros(rows, c, dtype=BF, device="cuda")
    at = list(range(3)) + list(range(rows - 70, rows))
    t[at] = torch.randn(len(at), c, generator=g).to(BF).cuda()
    return t, at


def close(got, want, tol):
    off = (got.double().cpu() - want).abs() - tol
    assert not torch.isnan(off).any() and off.max() <= 0, float(off.max())


@pytest.mark.parametrize("rows,c", [(70001, 32768), (2200003, 1000), (65539, 32776)])
def test_layer_norm(tbn, rows, c):
    x, at = rows_of(rows, c, 1)
    gamma, beta = torch.full((c,), 2.0, device="cuda"), torch.full((c,), 0.5, device="cuda")
    y, mean, inv_std = tbn.layernorm_fwd(x, gamma, beta)
    xd = x[at].double().cpu()
    mu = xd.mean(1, keepdim=True)
    s = 1 / ((xd - mu).square().mean(1, keepdim=True) + 1e-5).sqrt()
    want = (xd - mu) * s * 2 + 0.5
    # statistics within 64 roundings of numbers of size 1 (c up to 32776 in a thread's and a tree's sums), then the output's rounding
    close(y[at], want, 2.0 ** -8 * want.abs() + 1000 * U * (1 + want.abs()))
    assert float(y[rows // 2].float().min()) == float(y[rows // 2].float().max()) == 0.5
    del y
    dx, dgamma, dbeta = tbn.layernorm_bwd(x, x, mean, inv_std, gamma)
    xh = (xd - mu) * s
    h = xd * 2
    want = s * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    close(dx[at], want, 2.0 ** -8 * want.abs() + 1000 * U * (1 + h.abs()) * s)
    assert not dx[rows // 2].any()
    close(dgamma, (xd * xh).sum(0), 1000 * U * (1 + (xd * xh).abs().sum(0)))
    close(dbeta, xd.sum(0), 1000 * U * (1 + xd.abs().sum(0)))


def test_adapters(tbn):
    rows, c, k, rank = 70001, 32768, 64, 4
    g = torch.Generator().manual_seed(2)
    x, at = rows_of(rows, c, 3)
    index = torch.full((rows,), -1, dtype=torch.int32)
    index[at] = torch.randint(0, 12, (len(at),), generator=g).to(torch.int32)
    a, b = (torch.randn(12, rank, c, generator=g) * c ** -0.5).to(BF), torch.randn(12, k, rank, generator=g).to(BF)
    d = [t.cuda() for t in (index, a, b)]
    y, t = tbn.adapter_fwd(x, *d, out_dtype=torch.float32)
    xd, i = x[at].double().cpu(), index[at].long()
    want_t = torch.stack([a[n].double() @ v for n, v in zip(i, xd)])
    size = torch.stack([a[n].double().abs() @ v.abs() for n, v in zip(i, xd)])
    close(t[at], want_t, (c / 32 + 64) * U * size)
    want = torch.stack([b[n].double() @ v for n, v in zip(i, want_t)])
    close(y[at], want, torch.stack([b[n].double().abs() @ v for n, v in zip(i, (c / 32 + 200) * U * size)]))
    assert not y[rows // 2].any() and not t[rows // 2].any()
    # the other way round: dx of that size
    dy = torch.zeros(rows, k, dtype=BF, device="cuda")
    dy[at] = torch.randn(len(at), k, generator=g).to(BF).cuda()
    dx, da, db = tbn.adapter_bwd(x, dy, *d, t)
    dyd = dy[at].double().cpu()
    dt = torch.stack([v @ b[n].double() for n, v in zip(i, dyd)])
    dt_size = torch.stack([v.abs() @ b[n].double().abs() for n, v in zip(i, dyd)])
    want = torch.stack([v @ a[n].double() for n, v in zip(i, dt)])
    close(dx[at], want, 2.0 ** -8 * want.abs() + torch.stack([v @ a[n].double().abs() for n, v in zip(i, 200 * U * dt_size)]))
    assert not dx[rows // 2].any()
    own = torch.nn.functional.one_hot(i, 12).double()
    close(da, torch.einsum("nb,nr,nc->brc", own, dt, xd), 200 * U * torch.einsum("nb,nr,nc->brc", own, dt_size, xd.abs()) + 1e-300)
    td = t[at].double().cpu()
    close(db, torch.einsum("nb,nk,nr->bkr", own, dyd, td), 200 * U * torch.einsum("nb,nk,nr->bkr", own, dyd.abs(), td.abs()) + 1e-300)


def test_adamw(tbn):
    n, tail = (1 << 31) + 1027, 3000
    w, m, v, g = (torch.zeros(n, device="cuda") for _ in range(4))
    gen = torch.Generator().manual_seed(5)
    for t in (w, g):
        t[:tail] = torch.randn(tail, generator=gen).cuda()
        t[-tail:] = torch.randn(tail, generator=gen).cuda()
    parts = [torch.cat([t[:tail], t[-tail:]]).double().cpu() for t in (w, g)]
    tbn.adamw_step([w], [m], [v], [g], 1, lr=1e-2, weight_decay=0.1)
    # the first step moves by lr g / (|g| + eps)
    want = parts[0] * (1 - 1e-3) - 1e-2 * parts[1] / (parts[1].abs() + 1e-8)
    close(torch.cat([w[:tail], w[-tail:]]), want, 4 * U * parts[0].abs() + 2 * U * want.abs() + 30 * U * 1e-2)
    assert not w[n // 2 - 1000:n // 2 + 1000].any()
