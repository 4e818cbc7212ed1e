"""Operands that lie side by side in one buffer, an end at another's beginning: taken, with the same bits as apart (what overlaps by a
byte is refused: test_finetune_refusals.py)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


class Pack:
    """Tensors in turn in one buffer, in the given order, without gaps."""

    def __init__(self, **tensors):
        self.sizes = {n: t.numel() * t.element_size() for n, t in tensors.items()}
        flat = torch.empty(sum(self.sizes.values()), dtype=torch.uint8, device="cuda")
        at = 0
        for n, t in tensors.items():
            part = flat[at:at + self.sizes[n]].view(t.dtype).view(t.shape)
            part.copy_(t)
            setattr(self, n, part)
            at += self.sizes[n]


def equal(p, q):
    assert torch.equal(p.reshape(-1).view(torch.uint8), q.reshape(-1).view(torch.uint8))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(tbn, bits):
    n = 1024  # (bytes of every array a multiple of 16)
    g = torch.Generator().manual_seed(1)
    w, grad = torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()
    m, v, ms, vs = tbn.adamw_state(w, bits=bits)
    scales = {} if bits == 32 else {"ms": ms, "vs": vs}
    p = Pack(g=grad, w=w, m=m, g2=grad, v=v, **scales, w2=w, g3=grad)
    kw = {} if bits == 32 else {"m_scale": [p.ms], "v_scale": [p.vs]}
    kw2 = {} if bits == 32 else {"m_scale": [ms], "v_scale": [vs]}
    for step, name in ((1, "g"), (2, "g2"), (3, "g3")):
        tbn.adamw_step([p.w], [p.m], [p.v], [getattr(p, name)], step, **kw)
        tbn.adamw_step([w], [m], [v], [grad], step, **kw2)
    for a, b in ((p.w, w), (p.m, m), (p.v, v), (p.g, grad), (p.g3, grad)):
        equal(a, b)
    # one gradient of two tensors is taken, a gradient that is w itself is not
    w2 = p.w2.clone()
    st = [torch.zeros(n, device="cuda") for _ in range(4)]
    tbn.adamw_step([p.w2, w2], st[:2], st[2:], [p.g3, p.g3], 1)
    equal(p.w2, w2)
    with pytest.raises(tbn.TbnError, match="overlap"):
        tbn.adamw_step([p.w2], [st[0]], [st[1]], [p.w2], 1)


def test_layer_norm(tbn):
    g = torch.Generator().manual_seed(2)
    rows, c = 48, 72
    x, dy = torch.randn(rows, c, generator=g).to(BF).cuda(), torch.randn(rows, c, generator=g).to(BF).cuda()
    gamma, beta = torch.randn(c, generator=g).cuda(), torch.randn(c, generator=g).cuda()
    want = tbn.layernorm_fwd(x, gamma, beta)
    wanted = tbn.layernorm_bwd(x, dy, want[1], want[2], gamma)
    ws = torch.zeros(tbn.layernorm_workspace_size(rows, c), dtype=torch.uint8, device="cuda")
    p = Pack(dgamma=gamma, gamma=gamma, beta=beta, x=x, dy=dy, mean=want[1], inv_std=want[2], ws=ws, dbeta=beta)
    for a, b in zip(tbn.layernorm_fwd(p.x, p.gamma, p.beta), want):
        equal(a, b)
    for a, b in zip(tbn.layernorm_bwd(p.x, p.dy, p.mean, p.inv_std, p.gamma, ws=p.ws, dgamma=p.dgamma, dbeta=p.dbeta), wanted):
        equal(a, b)
    for bad in ({"dgamma": p.gamma}, {"dgamma": p.dgamma, "dbeta": p.dgamma}):
        with pytest.raises(tbn.TbnError, match="overlap"):
            tbn.layernorm_bwd(p.x, p.dy, p.mean, p.inv_std, p.gamma, **bad)


@pytest.mark.parametrize("rows,bank", [(48, 4), (320, 4), (1120, 12)])
def test_adapters(tbn, rows, bank):
    g = torch.Generator().manual_seed(3)
    c, k, rank = 64, 48, 8
    normal = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    index = torch.randint(-1, bank, (rows,), generator=g).to(torch.int32).cuda()
    x, dy, a, b = normal(rows, c).to(BF), normal(rows, k).to(BF), normal(bank, rank, c), normal(bank, k, rank)
    res, scale = normal(rows, k).to(BF), normal(bank)
    y, t = tbn.adapter_fwd(x, index, a, b, scale=scale, residual=res)
    grads = tbn.adapter_bwd(x, dy, index, a, b, t, scale=scale, residual=x)
    d = tbn.AdapterDesc(rows, c, k, rank, bank)
    ws = [torch.zeros(tbn.adapter_workspace_size(op, d), dtype=torch.uint8, device="cuda") for op in (tbn.OP_FWD, tbn.OP_BWD_DATA)]
    p = Pack(y=res, x=x, ws=ws[0], index=index, da=a, a=a, db=b, b=b, dy=dy, t=t, ws2=ws[1], scale=scale)
    out, t2 = tbn.adapter_fwd(p.x, p.index, p.a, p.b, scale=p.scale, residual=p.y, y=p.y, ws=p.ws)
    equal(out, y)
    equal(t2, t)
    for q, w in zip(tbn.adapter_bwd(p.x, p.dy, p.index, p.a, p.b, p.t, scale=p.scale, residual=p.x, da=p.da, db=p.db, ws=p.ws2), grads):
        equal(q, w)
    for bad in ({"da": p.a}, {"da": p.da, "db": p.da.view(-1)[:p.b.numel()].view_as(p.b)}):
        with pytest.raises(tbn.TbnError, match="overlap"):
            tbn.adapter_bwd(p.x, p.dy, p.index, p.a, p.b, p.t, **bad)
