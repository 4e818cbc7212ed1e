"""Frozen two-bit layers with adapters and a layer normalisation between them, trained by AdamW: the calls together
as they are used, eagerly, captured and on two streams at once, against the formulas in 64 bits; and the calls' native
marshalling against the ctypes code.

x (bf16) -> z1 = x W1~ + adapters -> y1 = bf16(layernorm(z1)) -> z2 = y1 W2~ + adapters, loss = sum(z2 dz2).

Tolerances: the net is linear but for the normalisation, whose input is fp32, so two roundings to bf16 (H = 2^-8 of the
value, half a step) reach the results, y1 and dz1, and a third may lie in the projection's backward pass (alpha dz2 as bf16).
Each goes on linearly: the bounds below are the formulas again with magnitudes in place of values.  fp32 sums of up to 192
products are off by (192 / 32 + 64) 2^-24 of the magnitudes' sum, which is below 20 times the result's typical size: 1e-4
(E) of a value's scale covers each of them.
"""
import pytest
import torch

from test_gpu_adamw import check_w
from test_gpu_binding import _Declines, _Recorder, _tensors

pytestmark = pytest.mark.gpu

H, E = 2.0 ** -8, 1e-4
BF, F = torch.bfloat16, torch.float32
C, M, K, RANK, BANK = 96, 192, 160, 8, 3


class Net:
    def __init__(self, tbn, rows, bits=32, seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, size=1.0):
            return (torch.randn(*shape, generator=g) * size).cuda()

        self.tbn, self.rows = tbn, rows
        self.x, self.dz = normal(rows, C).to(BF), normal(rows, K).to(BF)
        self.index = torch.repeat_interleave(torch.randint(-1, BANK, (rows,), generator=g), 5)[:rows].to(torch.int32).cuda()
        self.layers = [tbn.quantize(normal(n, c))[:2] for n, c in ((M, C), (K, M))]
        self.desc = [tbn.ConvDesc(rows, 1, 1, c, n, 1, 1) for n, c in ((M, C), (K, M))]
        self.scale = torch.tensor([0.5, 2.0, 1.0]).cuda()
        self.p = [normal(M, size=0.2) + 1, normal(M, size=0.1), normal(BANK, RANK, C, size=0.1), normal(BANK, M, RANK, size=0.3),
                  normal(BANK, RANK, M, size=0.1), normal(BANK, K, RANK, size=0.3)]
        s = [tbn.adamw_state(t, bits=bits) for t in self.p]
        self.m, self.v = [t[0] for t in s], [t[1] for t in s]
        self.scales = {} if bits == 32 else {"m_scale": [t[2] for t in s], "v_scale": [t[3] for t in s]}
        self.step = torch.ones(1, dtype=torch.int32, device="cuda")
        self.lr = torch.full((1,), 0.01, device="cuda")

    def forward_backward(self):
        tbn, (gamma, beta, a1, b1, a2, b2) = self.tbn, self.p
        z1 = tbn.conv2d_fwd(self.desc[0], self.x, *self.layers[0], out_dtype=F).view(self.rows, M)
        z1, t1 = tbn.adapter_fwd(self.x, self.index, a1, b1, scale=self.scale, residual=z1, y=z1)
        y1, mean, inv_std = tbn.layernorm_fwd(z1, gamma, beta, out_dtype=BF)
        z2 = tbn.conv2d_fwd(self.desc[1], y1, *self.layers[1], out_dtype=F).view(self.rows, K)
        z2, t2 = tbn.adapter_fwd(y1, self.index, a2, b2, scale=self.scale, residual=z2)
        dy1 = tbn.conv2d_bwd_data(self.desc[1], self.dz, *self.layers[1], out_dtype=F).view(self.rows, M)
        dy1, da2, db2 = tbn.adapter_bwd(y1, self.dz, self.index, a2, b2, t2, scale=self.scale, residual=dy1, out_dtype=F)
        dz1, dgamma, dbeta = tbn.layernorm_bwd(z1, dy1, mean, inv_std, gamma)
        _, da1, db1 = tbn.adapter_bwd(self.x, dz1.to(BF), self.index, a1, b1, t1, scale=self.scale, need_dx=False)
        return z2, [dgamma, dbeta, da1, db1, da2, db2]

    def train(self):
        out = self.forward_backward()
        self.tbn.adamw_step(self.p, self.m, self.v, out[1], self.step, lr=self.lr, weight_decay=[0.0, 0.0] + [0.1] * 4, seed=3,
                            **self.scales)
        self.step.add_(1)
        return out

    def state(self):
        return [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in self.p + self.m + self.v] + \
            [t for s in self.scales.values() for t in s]

    def dense(self, k):
        # W~ of a layer: its outputs for unit vectors
        codes, alpha = self.layers[k]
        c = self.desc[k].c
        eye = torch.eye(c, device="cuda").to(BF)
        return self.tbn.conv2d_fwd(self.tbn.ConvDesc(c, 1, 1, c, self.desc[k].k, 1, 1), eye, codes, alpha,
                                   out_dtype=F).view(c, -1).double().cpu()


def expect(net):
    """What the net's results are in 64 bits, and how far off they may be."""
    x, dz, scale = net.x.double().cpu(), net.dz.double().cpu(), net.scale.double().cpu()
    gamma, beta, a1, b1, a2, b2 = (t.double().cpu() for t in net.p)
    w1, w2, index = net.dense(0), net.dense(1), net.index.cpu().long()
    has = (index >= 0).double()[:, None]
    i = index.clamp(min=0)
    sc = scale[i][:, None] * has

    def rows(v, w):  # row r times its own matrix
        return torch.stack([v[r] @ w[i[r]] for r in range(len(i))])

    def bank(v, u):  # sums over each adapter's rows of outer products
        own = torch.nn.functional.one_hot(i, BANK).double() * has
        return torch.stack([(v * own[:, k:k + 1]).t() @ u for k in range(BANK)])

    tr = lambda w: w.transpose(1, 2)  # noqa: E731
    t1 = rows(x, tr(a1))
    z1 = x @ w1 + sc * rows(t1, tr(b1))
    mean = z1.mean(1, keepdim=True)
    s = 1 / ((z1 - mean).square().mean(1, keepdim=True) + 1e-5).sqrt()
    xh = (z1 - mean) * s
    y1 = xh * gamma + beta
    e_y1 = H * y1.abs() + 2 * E * (1 + xh.abs()) * gamma.abs()
    t2 = rows(y1, tr(a2))
    e_t2 = rows(e_y1, tr(a2).abs())
    z2 = y1 @ w2 + sc * rows(t2, tr(b2))
    e_z2 = e_y1 @ w2.abs() + sc * rows(e_t2, tr(b2).abs()) + E * (y1.abs() @ w2.abs() + sc * rows(t2.abs(), tr(b2).abs()))
    dt2 = sc * rows(dz, b2)
    e_dt2 = E * sc * rows(dz.abs(), b2.abs())
    dy1 = dz @ w2.t() + rows(dt2, a2)
    e_dy1 = (H + E) * (dz.abs() @ w2.t().abs()) + rows(e_dt2 + E * dt2.abs(), a2.abs())
    h, e_h = dy1 * gamma, e_dy1 * gamma.abs() + E * (dy1 * gamma).abs()
    dz1 = s * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    e_dz1 = s * (e_h + e_h.mean(1, keepdim=True) + xh.abs() * (e_h * xh.abs()).mean(1, keepdim=True)) + H * dz1.abs() + \
        4 * E * s * (1 + xh.abs()) * h.abs().mean(1, keepdim=True)
    dt1 = sc * rows(dz1, b1)
    e_dt1 = sc * rows(e_dz1, b1.abs())
    e_xh = 2 * E * (1 + xh.abs())
    want = [(dy1 * xh).sum(0), dy1.sum(0), bank(dt1, x), bank(dz1, sc * t1), bank(dt2, y1), bank(dz, sc * t2)]
    tol = [(e_dy1 * xh.abs() + dy1.abs() * e_xh).sum(0), e_dy1.sum(0) + E * dy1.abs().sum(0),
           bank(e_dt1 + E * dt1.abs(), x.abs()), bank(e_dz1 + E * dz1.abs(), sc * t1.abs()),
           bank(e_dt2 + E * dt2.abs(), y1.abs()) + bank(dt2.abs(), e_y1), bank(dz.abs(), sc * (e_t2 + E * t2.abs()))]
    return z2, e_z2, want, tol


def close(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol - 1e-300
    assert not torch.isnan(off).any() and off.max() <= 0, "%s: %g over the tolerance" % (what, off.max())


@pytest.mark.parametrize("rows", [1, 30, 64, 65, 300])
def test_forward_and_gradients(tbn, rows):
    net = Net(tbn, rows, seed=rows)
    z2, grads = net.forward_backward()
    want_z, tol_z, want, tol = expect(net)
    close(z2, want_z, tol_z, "z2")
    for name, g, w, t in zip(("dgamma", "dbeta", "da1", "db1", "da2", "db2"), grads, want, tol):
        close(g, w, t, name)


def test_a_step_of_all_parameters(tbn):
    net = Net(tbn, 70)
    before = [t.cpu() for t in net.p]
    _, grads = net.train()
    for k, (p, w0, g) in enumerate(zip(net.p, before, grads)):
        zero = torch.zeros_like(w0)
        check_w(p, w0, zero, zero, g.cpu(), 1, 0.1 if k > 1 else 0.0,
                {"lr": float(torch.tensor(0.01)), "beta1": 0.9, "beta2": 0.999, "eps": 1e-8})


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows", [33, 260])
def test_captured_training_equals_eager(tbn, bits, rows):
    eager, net = Net(tbn, rows, bits), Net(tbn, rows, bits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = net.train()
    for k in range(4):
        other = Net(tbn, rows, bits, seed=10 + k)  # other rows, targets and requests
        for n in (eager, net):
            n.x.copy_(other.x)
            n.dz.copy_(other.dz)
            n.index.copy_(other.index)
            n.lr.fill_(0.01 / (k + 1))
        want = eager.train()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and all(torch.equal(a, b) for a, b in zip(out[1], want[1]))
        assert int(net.step) == k + 2
        assert all(torch.equal(a, b) for a, b in zip(net.state(), eager.state()))


def test_two_streams_at_once(tbn):
    nets = [Net(tbn, 300, 8, seed=5), Net(tbn, 48, 8, seed=6)]
    alone = [Net(tbn, 300, 8, seed=5), Net(tbn, 48, 8, seed=6)]
    for n in alone:
        for _ in range(3):
            n.train()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for n, s in zip(nets, streams):
            with torch.cuda.stream(s):
                n.train()
    torch.cuda.synchronize()
    for n, a in zip(nets, alone):
        assert all(torch.equal(p, q) for p, q in zip(n.state(), a.state()))


def test_two_graphs_one_workspace(tbn):
    # replayed in turn on one stream; each call leaves nothing in its workspace that another needs
    n = Net(tbn, 90)
    a, b = n.p[2], n.p[3]
    dy = torch.randn(90, M, device="cuda").to(BF)
    z = torch.randn(90, C, device="cuda")
    gamma = torch.rand(C, device="cuda") + 0.5
    _, mean, inv_std = tbn.layernorm_fwd(z, gamma)
    need = max(tbn.adapter_workspace_size(op, tbn.AdapterDesc(90, C, M, RANK, BANK)) for op in (tbn.OP_FWD, tbn.OP_BWD_DATA))
    ws = torch.empty(max(need, tbn.layernorm_workspace_size(90, C)), dtype=torch.uint8, device="cuda")

    def first():
        y, t = tbn.adapter_fwd(n.x, n.index, a, b, ws=ws)
        return (y, t) + tbn.adapter_bwd(n.x, dy, n.index, a, b, t, ws=ws)

    def second():
        return tbn.layernorm_bwd(z, z, mean, inv_std, gamma, ws=ws)

    want = [first(), second()]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f in (first, second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(f())
        graphs.append(g)
    for _ in range(3):
        ws.fill_(255)  # NaN to every reader
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(p, q) for p, q in zip(o, w))


def calls(tbn):
    n = Net(tbn, 70)
    gamma, beta, a, b = n.p[:4]
    z = torch.randn(70, M, device="cuda")
    dy = torch.randn(70, M, device="cuda").to(BF)
    _, mean, inv_std = tbn.layernorm_fwd(z, gamma, beta)
    y0, t = tbn.adapter_fwd(n.x, n.index, a, b)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def adamw(bits, gt=F, step=2, lr=1e-3, decay=0.01):
        w = [x.clone() for x in n.p]
        s = [tbn.adamw_state(x, bits=bits) for x in w]
        kw = {} if bits == 32 else {"m_scale": [x[2] for x in s], "v_scale": [x[3] for x in s], "seed": 7}
        p, m, v = tbn.adamw_step(w, [x[0] for x in s], [x[1] for x in s], [(x * 0.1).to(gt) for x in n.p], step, lr=lr,
                                 weight_decay=decay, **kw)
        return p, [x.view(torch.uint8) for x in m], [x.view(torch.uint8) for x in v], kw.get("m_scale"), kw.get("v_scale")

    return {
        "ln": lambda: tbn.layernorm_fwd(z, gamma, beta),
        "ln plain": lambda: tbn.layernorm_fwd(z, out_dtype=BF, want_stats=False),
        "ln bwd": lambda: tbn.layernorm_bwd(z, dy, mean, inv_std, gamma),
        "ln bwd given": lambda: tbn.layernorm_bwd(z, z, mean, inv_std, None, ws=ws, dgamma=torch.empty(M, device="cuda"),
                                                  dbeta=torch.empty(M, device="cuda")),
        "adapter": lambda: tbn.adapter_fwd(n.x, n.index, a, b, scale=n.scale, residual=dy),
        "adapter y": lambda: tbn.adapter_fwd(n.x, n.index, a, b, residual=z, y=torch.empty_like(z), want_t=False, ws=ws),
        "adapter bf16": lambda: tbn.adapter_fwd(n.x, n.index, a.to(BF), b.to(BF), out_dtype=F),
        "adapter bwd": lambda: tbn.adapter_bwd(n.x, dy, n.index, a, b, t, scale=n.scale, residual=n.x),
        "adapter bwd no dx": lambda: tbn.adapter_bwd(n.x, dy, n.index, a, b, t, need_dx=False, da=torch.empty_like(a),
                                                     db=torch.empty_like(b), ws=ws),
        "adamw": lambda: adamw(32),
        "adamw 8": lambda: adamw(8, BF, decay=[0.1] * 6),
        "adamw device step": lambda: adamw(8, F, torch.full((1,), 9, dtype=torch.int32, device="cuda"),
                                           torch.full((1,), 0.1, device="cuda")),
    }, {
        "ln cpu": lambda: tbn.layernorm_fwd(z.cpu(), gamma, beta),
        "ln strided": lambda: tbn.layernorm_fwd(z.t(), gamma),
        "ln gamma": lambda: tbn.layernorm_fwd(z, gamma[:5], beta),
        "ln type": lambda: tbn.layernorm_fwd(z.half()),
        "ln bwd size": lambda: tbn.layernorm_bwd(z, dy[:3], mean, inv_std, gamma),
        "ln workspace": lambda: tbn.layernorm_bwd(z, dy, mean, inv_std, gamma, ws=small),
        "adapter index": lambda: tbn.adapter_fwd(n.x, n.index.long(), a, b),
        "adapter bank": lambda: tbn.adapter_fwd(n.x, n.index, a, b[:2]),
        "adapter weights": lambda: tbn.adapter_fwd(n.x, n.index, a, b.to(BF)),
        "adapter residual": lambda: tbn.adapter_fwd(n.x, n.index, a, b, residual=z[:3]),
        "adapter workspace": lambda: tbn.adapter_bwd(n.x, dy, n.index, a, b, t, ws=small),
        "adamw lists": lambda: tbn.adamw_step([gamma], [beta, beta], [gamma], [gamma], 1),
        "adamw types": lambda: tbn.adamw_step([gamma], [gamma.to(BF)], [gamma], [gamma], 1),
        "adamw scales": lambda: tbn.adamw_step([gamma], [gamma], [gamma], [gamma], 1, m_scale=[beta], v_scale=[beta]),
        "adamw step": lambda: tbn.adamw_step([gamma.clone()], [beta.clone()], [beta.abs()], [gamma], 0),
    }


def test_native_calls_equal_ctypes_calls(tbn, monkeypatch):
    ordinary, refused = calls(tbn)
    monkeypatch.setattr(tbn, "_native", None)

    def outcome(f):
        try:
            return _tensors(f())
        except Exception as e:  # the type and the message are compared
            return (type(e), str(e))

    module = tbn._load_native()
    for name, f in list(ordinary.items()) + list(refused.items()):
        print(name, flush=True)
        recorder = _Recorder(module)
        monkeypatch.setattr(tbn, "_native", recorder)
        got = outcome(f)
        took = (recorder.answered, recorder.declined)
        monkeypatch.setattr(tbn, "_native", _Declines())
        want = outcome(f)
        if name in refused:
            assert isinstance(want, tuple) and got == want, (name, got, want)
            continue
        assert took == (1, 0), (name, took)
        assert not isinstance(got, tuple), (name, got)
        assert [(t.shape, t.dtype) for t in got] == [(t.shape, t.dtype) for t in want]
        assert all(torch.equal(s, t) for s, t in zip(got, want)), name
