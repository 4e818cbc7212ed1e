"""A feed-forward block of two-bit layers, trained by Muon on its real weights, with an 8-bit layer behind it: the calls together as they are
used, eagerly, captured, on two streams at once, on one workspace; and their native marshalling against the ctypes code.

x (bf16) -> h = act(g) u of W1~ [2 F][C] -> z = h W2~ [C][F] -> y = z W3 in 8 bits; loss = sum(z dz), the gradients straight-through.
"""
import pytest
import torch

from test_gpu_binding import _Declines, _Recorder, _tensors
from test_gpu_glu import act64

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
H = 2.0 ** -8


class Net:
    def __init__(self, tbn, rows, c=96, f=80, n=50, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.tbn, self.rows, self.c, self.f = tbn, rows, c, f
        self.x, self.dz = (torch.randn(rows, c, generator=g).to(BF).cuda() for _ in range(2))
        self.w = [torch.randn(2 * f, c, generator=g).cuda(), torch.randn(c, f, generator=g).cuda()]
        self.m = [torch.zeros_like(t) for t in self.w]
        self.g = [torch.zeros_like(t) for t in self.w]
        self.lr = torch.full((1,), 0.1, device="cuda")
        self.last = tbn.quantize_rows_i8(torch.randn(n, c, generator=g).cuda())
        self.ws = torch.zeros(tbn.muon_workspace_size(self.w), dtype=torch.uint8, device="cuda")

    def forward(self, want_gu=False):
        tbn, rows, c, f = self.tbn, self.rows, self.c, self.f
        self.codes = [tbn.quantize(w)[:2] for w in self.w]
        h, gu = tbn.glu_fwd(self.x, *self.codes[0], want_gu=want_gu)
        z = tbn.conv2d_fwd(tbn.ConvDesc(rows, 1, 1, f, c, 1, 1), h, *self.codes[1]).view(rows, c)
        q, s = tbn.quantize_rows_i8(z)
        y = tbn.matmul_i8(q, s, *self.last, out_dtype=F)
        return h, gu, z, y

    def train(self, kept=True):
        tbn, rows, c, f = self.tbn, self.rows, self.c, self.f
        h, gu, z, y = self.forward(kept)
        down, up = tbn.ConvDesc(rows, 1, 1, f, c, 1, 1), tbn.ConvDesc(rows, 1, 1, c, 2 * f, 1, 1)
        dh = tbn.conv2d_bwd_data(down, self.dz, *self.codes[1]).view(rows, f)
        if kept:
            dgu, h2 = tbn.glu_bwd(dh, gu=gu, want_h=True)
        else:
            dgu, h2 = tbn.glu_bwd(dh, x=self.x, codes=self.codes[0][0], alpha=self.codes[0][1], want_h=True)
        tbn.conv2d_bwd_weight(up, self.x, dgu, dw=self.g[0])
        tbn.conv2d_bwd_weight(down, h2, self.dz, dw=self.g[1])
        dx = tbn.conv2d_bwd_data(up, dgu, *self.codes[0]).view(rows, c)
        tbn.muon_step(self.w, self.m, self.g, lr=self.lr, weight_decay=0.01, ws=self.ws)
        return h, z, y, dx

    def state(self):
        return [t.clone() for t in self.w + self.m + self.g]


def same(a, b):
    return len(a) == len(b) and all(torch.equal(s, t) for s, t in zip(a, b))


def test_a_step_against_the_formulas(tbn):
    for kept in (True, False):
        net = Net(tbn, 70)
        w0 = [w.double() for w in net.w]
        net.train(kept)
        values = [torch.where(w > 0, 1.0, -1.0).double() * torch.where(w.abs() > 1, 2.0, 1.0) * a.double()[:, None]
                  for w, (_, a) in zip(w0, net.codes)]
        x, dz = net.x.double(), net.dz.double()
        g, u = (x @ values[0].t()).chunk(2, 1)
        a, slope = act64("silu", g)
        h, dh = a * u, dz @ values[1]
        dgu = torch.cat([dh * u * slope, dh * a], 1)
        # each of g, u, h, dh, alpha and dgu is rounded to bf16 at most once (H of its value; |act'| <= 1.13, |act''| <= 0.5), and what the
        # fp32 sums lose is below 1e-4 of their magnitudes
        t = H + 1e-4
        e_g, e_u = t * g.abs(), t * u.abs()
        e_h = t * h.abs() + 1.13 * e_g * (u.abs() + e_u) + a.abs() * e_u
        e_dh = 2 * t * (dz.abs() @ values[1].abs())
        e_dg = t * dgu[:, :net.f].abs() + e_dh * (u * slope).abs() + (dh.abs() + e_dh) * (e_u * (slope.abs() + 0.5 * e_g) + u.abs() * 0.5 * e_g)
        e_du = t * dgu[:, net.f:].abs() + e_dh * a.abs() + (dh.abs() + e_dh) * 1.13 * e_g
        want = [dgu.t() @ x, dz.t() @ h]
        bound = [torch.cat([e_dg, e_du], 1).t() @ x.abs() + 1e-4 * (dgu.abs().t() @ x.abs()), dz.abs().t() @ e_h + 1e-4 * (dz.abs().t() @ h.abs())]
        for got, v, e in zip(net.g, want, bound):
            assert ((got.double() - v).abs() <= 1.01 * e + 1e-6).all()
        # and the weights have moved along orthogonal updates: singular values of (w0 (1 - lr wd) - w) / lr / scale around 1
        for w, v in zip(net.w, w0):
            move = (v * (1 - 0.1 * 0.01) - w.double()) / 0.1 / max(1.0, w.shape[0] / w.shape[1]) ** 0.5
            s = torch.linalg.svdvals(move)
            assert s.max() < 1.25 and s.median() > 0.6


def test_captured_steps(tbn):
    """Replays with the program's own work and synchronisations between them, two graphs on one workspace."""
    eager, nets = Net(tbn, 300), [Net(tbn, 300), Net(tbn, 300, seed=1)]
    other = Net(tbn, 300, seed=1)
    for n in nets:
        n.ws = nets[0].ws
    side, graphs, outs = torch.cuda.Stream(), [], []
    before = [n.state() for n in nets]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for n in nets:
            n.train()
    torch.cuda.current_stream().wait_stream(side)
    for n, b in zip(nets, before):
        for t, s in zip(n.w + n.m + n.g, b):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(n.train())
        graphs.append(graph)
    for step in range(5):
        lr = 0.1 / (step + 1)
        for n in nets + [eager, other]:
            n.lr.fill_(lr)
        for graph, out, ref, n in zip(graphs, outs, (eager, other), nets):
            graph.replay()
            want = ref.train()
            torch.cuda.synchronize()
            assert same(out, want), step
            assert same(n.state(), ref.state()), step
        torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")


def test_two_streams_at_once(tbn):
    nets, refs = [Net(tbn, r, seed=s) for s, r in ((0, 300), (1, 70))], [Net(tbn, r, seed=s) for s, r in ((0, 300), (1, 70))]
    streams = [torch.cuda.Stream() for _ in nets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for n, s in zip(nets, streams):
            with torch.cuda.stream(s):
                n.train()
    torch.cuda.synchronize()
    for n, r in zip(nets, refs):
        for _ in range(4):
            r.train()
    torch.cuda.synchronize()
    assert all(same(n.state(), r.state()) for n, r in zip(nets, refs))


def test_serving_one_token_is_the_batch_within_rounding(tbn):
    """Rows of a batch and the same rows alone go through other kernels: the same sums in another order."""
    net = Net(tbn, 200, c=520, f=400)
    h, _, z, y = net.forward()
    for i in (0, 117, 199):
        h1, _ = tbn.glu_fwd(net.x[i:i + 1], *net.codes[0])
        assert ((h1.double() - h[i:i + 1].double()).abs() <= 2 * H * h[i].double().abs() + 1e-2).all()
        q, s = tbn.quantize_rows_i8(z[i:i + 1])
        assert torch.equal(tbn.matmul_i8(q, s, *net.last, out_dtype=F), y[i:i + 1])  # exact sums: the same bits


@pytest.mark.parametrize("rows", [1, 16])
def test_captured_tokens(tbn, rows):
    """A serving step of few rows, captured: its replays over new tokens are the eager step's bits."""
    nets = [Net(tbn, rows, c=1000, f=333), Net(tbn, rows, c=1000, f=333)]
    for n in nets:
        n.forward(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nets[0].forward(True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = nets[0].forward(True)
    for step in range(5):
        x = torch.randn(nets[0].x.shape, device="cuda").to(BF)
        for n in nets:
            n.x.copy_(x)
        graph.replay()
        want = nets[1].forward(True)
        torch.cuda.synchronize()
        assert same(out, want), step


@pytest.mark.parametrize("rows,c,f", [(1, 64, 7), (3, 500, 33), (16, 4200, 100), (5, 8300, 43), (20, 600, 45), (70, 100, 4100), (70, 2100, 3999), (900, 72, 1333), (1500, 72, 1601)])
def test_nothing_is_written_behind_an_output(tbn, rows, c, f):
    """Rows of odd lengths are written 16 bytes at a time: what lies before an output's first value and behind its last stays as it was."""
    x = torch.randn(rows, c, device="cuda").to(BF)
    codes, alpha = tbn.quantize(torch.randn(2 * f, c, device="cuda"))[:2]
    dh = torch.randn(rows, f, device="cuda").to(BF)

    def within(n, dtype, call):
        buf = torch.full((n + 128,), -7.0, device="cuda", dtype=dtype)
        out = buf[64:64 + n]
        call(out)
        assert (buf[:64] == -7).all() and (buf[64 + n:] == -7).all()
        return out.clone()

    for dtype in (BF, F):
        h = within(rows * f, dtype, lambda o: tbn.glu_fwd(x, codes, alpha, h=o.view(rows, f)))
        assert same([h.view(rows, f)], [tbn.glu_fwd(x, codes, alpha, out_dtype=dtype)[0]])
    gu = tbn.glu_fwd(x, codes, alpha, want_gu=True)[1]
    for kw in ({"gu": gu}, {"x": x, "codes": codes, "alpha": alpha}):
        dgu = within(rows * 2 * f, BF, lambda o: tbn.glu_bwd(dh, dgu=o.view(rows, 2 * f), **kw))
        assert same([dgu.view(rows, 2 * f)], [tbn.glu_bwd(dh, **kw)[0]])
    q, s = tbn.quantize_rows_i8(x)
    wq, ws = tbn.quantize_rows_i8(torch.randn(f, c, device="cuda"))
    for dtype in (BF, F):
        res = torch.randn(rows, f, device="cuda").to(dtype)
        y = within(rows * f, dtype, lambda o: tbn.matmul_i8(q, s, wq, ws, residual=res, y=o.view(rows, f)))
        assert same([y.view(rows, f)], [tbn.matmul_i8(q, s, wq, ws, residual=res, out_dtype=dtype)])


def _calls(tbn):
    net = Net(tbn, 20)
    codes, alpha = tbn.quantize(net.w[0])[:2]
    x, dh = net.x, torch.randn(20, net.f, device="cuda").to(BF)
    h, gu = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    q, s = tbn.quantize_rows_i8(x)
    wq, wsc = net.last
    bias, res = torch.randn(50, device="cuda"), torch.randn(20, 50, device="cuda").to(BF)
    fresh = lambda: [[t.clone() for t in l] for l in (net.w, net.m, [torch.ones_like(t) for t in net.w])]  # noqa: E731

    def muon(**kw):
        w, m, g = fresh()
        tbn.muon_step(w, m, kw.pop("g", g), **kw)
        return w, m

    lr = torch.full((1,), 0.3, device="cuda")
    ordinary = {
        "glu": lambda: tbn.glu_fwd(x, codes, alpha),
        "glu gu": lambda: tbn.glu_fwd(x.view(4, 5, -1), codes, alpha, act="gelu", want_gu=True, out_dtype=F),
        "glu into": lambda: tbn.glu_fwd(x, codes, alpha, h=torch.empty(20, net.f, device="cuda")),
        "glu bwd": lambda: tbn.glu_bwd(dh, gu=gu),
        "glu bwd x": lambda: tbn.glu_bwd(dh, x=x, codes=codes, alpha=alpha, act="relu", want_h=True, out_dtype=F),
        "muon": lambda: muon(),
        "muon all": lambda: muon(lr=lr, momentum=0.5, nesterov=False, weight_decay=[0.1, 0.2], scale=[1.0, 2.0], eps=1e-3, steps=3),
        "muon bf16": lambda: muon(g=[torch.ones_like(t).to(BF) for t in net.w], weight_decay=0.1),
        "rows": lambda: tbn.quantize_rows_i8(x),
        "rows into": lambda: tbn.quantize_rows_i8(x.float(), q=torch.empty(20, 96, dtype=torch.int8, device="cuda"), scale=torch.empty(20, device="cuda")),
        "matmul": lambda: tbn.matmul_i8(q, s, wq, wsc),
        "matmul all": lambda: tbn.matmul_i8(q, s, wq, wsc, scale=bias, bias=bias, residual=res, relu=True),
        "matmul into": lambda: tbn.matmul_i8(q, s, wq, wsc, y=torch.empty(20, 50, device="cuda")),
    }
    refused = {
        "act": lambda: tbn.glu_fwd(x, codes, alpha, act="tanh"),
        "codes": lambda: tbn.glu_fwd(x, codes[:-1], alpha),
        "alpha": lambda: tbn.glu_fwd(x, codes, alpha[:-1]),
        "x type": lambda: tbn.glu_fwd(x.float(), codes, alpha),
        "x strided": lambda: tbn.glu_fwd(x[:, ::2], codes, alpha),
        "h type": lambda: tbn.glu_fwd(x, codes, alpha, out_dtype=torch.float16),
        "gu size": lambda: tbn.glu_bwd(dh, gu=gu[:-1]),
        "no gu": lambda: tbn.glu_bwd(dh, x=x),
        "m size": lambda: tbn.muon_step(net.w, [net.m[0], net.m[0]], net.g),
        "mixed gradients": lambda: tbn.muon_step(net.w, net.m, [net.g[0], net.g[1].to(BF)]),
        "w type": lambda: tbn.muon_step([w.to(BF) for w in net.w], net.m, net.g),
        "c differs": lambda: tbn.matmul_i8(q, s, wq[:, :80].contiguous(), wsc),
        "residual type": lambda: tbn.matmul_i8(q, s, wq, wsc, residual=res, out_dtype=F),
        "scales": lambda: tbn.matmul_i8(q, s[:-1], wq, wsc),
    }
    library = {
        "misaligned": lambda: tbn.glu_fwd(torch.zeros(20 * 96 + 1, dtype=BF, device="cuda")[1:].view(20, 96), codes, alpha),
        "momentum": lambda: muon(momentum=1.0),
        "overlap": lambda: tbn.muon_step(net.w, net.w, net.g),
        "small workspace": lambda: muon(ws=torch.empty(100, dtype=torch.uint8, device="cuda")),
        "uneven c": lambda: tbn.matmul_i8(q[:, :90].contiguous(), s, wq[:, :90].contiguous(), wsc),
    }
    return ordinary, refused, library


def test_native_and_ctypes_calls_are_the_same(tbn, monkeypatch):
    ordinary, refused, library = _calls(tbn)

    def outcome(f):
        try:
            return _tensors(f())
        except Exception as e:  # the type and the message are compared
            return (type(e), str(e))

    native, module = {}, tbn._load_native()
    for calls in (ordinary, refused, library):
        for name, f in calls.items():
            recorder = _Recorder(module)
            monkeypatch.setattr(tbn, "_native", recorder)
            native[name] = outcome(f)
            took = (recorder.answered, recorder.declined)
            assert took == ((0, 1) if calls is refused else (1, 0)), (name, took)
    monkeypatch.setattr(tbn, "_native", _Declines())
    for calls in (ordinary, refused, library):
        for name, f in calls.items():
            print(name, flush=True)
            got, want = native[name], outcome(f)
            if calls is not ordinary:
                assert isinstance(want, tuple) and got == want, name
                continue
            assert not isinstance(got, tuple), got
            assert [(t.shape, t.dtype) for t in got] == [(t.shape, t.dtype) for t in want]
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name
