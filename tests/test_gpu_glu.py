"""The gated block of two-bit filters against its formulas in 64 bits, on every kernel: few rows (x in registers or read with the codes,
one or several groups of gates a block), tiles of four sizes, waves in groups, kept projections.

Tolerances.  A projection is a sum of c exact products in fp32, whose every addition is off by at most a step (2^-23 of the sum of the
magnitudes s = alpha sum |x w|), times alpha: e = (c + 2) 2^-23 s.  |act'| <= 1.13 and |act''| <= 0.8 for silu and gelu (1 and 0 for relu),
and the activation itself, its exponential and quotient or error function in fp32, is off by at most 2^-20 (1 + |g|), likewise its
slope.  What is rounded to bf16 is off by 2^-8 of its value, half a step.  relu's slope may be either one where |g| <= e.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
H, A = 2.0 ** -8, 2.0 ** -20


def block(tbn, rows, c, f, seed=0):
    g = torch.Generator().manual_seed(seed * 1000003 + rows * 31 + c * 7 + f)
    x = torch.randn(rows, c, generator=g).to(BF).cuda()
    on_gpu = torch.Generator("cuda").manual_seed(seed + rows + c + f)
    w = torch.randn(2 * f, c, generator=on_gpu, device="cuda")
    w[torch.rand(2 * f, c, generator=on_gpu, device="cuda") < 0.1] = 0.0  # code -1
    codes, alpha, _ = tbn.quantize(w)
    dh = torch.randn(rows, f, generator=g).to(BF).cuda()
    values = torch.where(w > 0, 1.0, -1.0).double() * torch.where(w.abs() > 1, 2.0, 1.0)
    return x, codes, alpha, dh, (values * alpha.double()[:, None])


def act64(name, g):
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        phi = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g.clamp(min=0), (g > 0).double()


def expect(x, w, act, dh=None, gu=None):
    """(gu, h, dgu) in 64 bits and how far off each may be, before its last rounding."""
    f = (w if gu is None else gu.t()).shape[0] // 2
    if gu is None:
        x64 = x.double()
        gu64, e = x64 @ w.t(), (w.shape[1] + 2) * 2.0 ** -23 * (x64.abs() @ w.t().abs())
    else:
        gu64, e = gu.double(), torch.zeros_like(gu, dtype=torch.float64)
    g, u, eg, eu = gu64[:, :f], gu64[:, f:], e[:, :f], e[:, f:]
    a, slope = act64(act, g)
    ea = 1.13 * eg + A * (1 + g.abs())
    es = (0.8 * eg if act != "relu" else (g.abs() <= eg).double()) + (A * (1 + g.abs()) if act != "relu" else 0)
    h, eh = a * u, a.abs() * eu + ea * (u.abs() + eu) + 2.0 ** -23 * (a * u).abs()
    if dh is None:
        return gu64, e, h, eh, None, None
    d = dh.double()
    dgu = torch.cat([d * u * slope, d * a], 1)
    edgu = torch.cat([d.abs() * (u.abs() * es + eu * (slope.abs() + es)), d.abs() * ea], 1) + 2.0 ** -22 * dgu.abs()
    return gu64, e, h, eh, dgu, edgu


def check(got, want, err, what):
    rounding = H if got.dtype == BF else 2.0 ** -24
    off = (got.double() - want).abs() - (err + rounding * (want.abs() + err) + 1e-38)
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), what
    assert off.max().item() <= 0, (what, off.max().item())


# rows, c, f: and the kernel that takes them
SHAPES = [
    (1, 1, 1), (1, 8, 3), (2, 7, 8), (3, 64, 16), (4, 100, 33), (1, 512, 1024),                       # few, x in registers: as it lies
    (5, 65, 31), (16, 128, 100), (9, 1000, 64), (16, 4090, 70),                                       # ... turned
    (16, 321, 8200), (16, 136, 16400), (1, 72, 16392), (6, 2100, 16500),                              # ... several groups a block
    (4, 5000, 40), (16, 8190, 33), (7, 4104, 4200), (5, 4200, 8300),                                  # ... two steps a wave
    (1, 24584, 20), (16, 8200, 100), (4, 13000, 17), (2, 8200, 8200), (3, 8200, 12300),               # ... x with the codes
    (17, 63, 1), (17, 8, 64), (40, 200, 40), (33, 256, 129), (150, 328, 4000), (320, 264, 4000), (777, 264, 1333),  # tiles of 64 x 64
    (150, 2056, 4000), (65, 2500, 4200),                                                              # ... in groups of waves
    (40, 512, 100), (64, 520, 31), (17, 4100, 65), (130, 2000, 32), (65, 1001, 4000),                 # 64 x 32 in groups of waves
    (1000, 130, 2000), (300, 513, 4500),                                                              # 128 x 64
    (4100, 72, 1601), (3300, 200, 2048), (1290, 1100, 2050),                                          # 128 x 128
]


@pytest.mark.parametrize("rows,c,f", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_forward_and_backward(tbn, rows, c, f, act):
    x, codes, alpha, dh, w = block(tbn, rows, c, f)
    gu64, e, h64, eh, dgu64, edgu = expect(x, w, act, dh)
    h, gu = tbn.glu_fwd(x, codes, alpha, act=act, want_gu=True)
    check(gu, gu64, e, "gu")
    check(h, h64, eh, "h")
    h32, none = tbn.glu_fwd(x, codes, alpha, act=act, out_dtype=F)
    assert none is None
    check(h32, h64, eh, "h in fp32")
    # without the kept projections: the same sums, so the same h as the forward pass
    dgu, again = tbn.glu_bwd(dh, x=x, codes=codes, alpha=alpha, act=act, want_h=True)
    check(dgu, dgu64, edgu, "dgu")
    assert torch.equal(again, h)
    # from the kept ones, rounded to bf16 as they are
    _, _, h64, eh, dgu64, edgu = expect(x, w, act, dh, gu=gu)
    dgu, h2 = tbn.glu_bwd(dh, gu=gu, act=act, want_h=True, out_dtype=F)
    check(dgu, dgu64, edgu, "dgu from gu")
    check(h2, h64, eh, "h from gu")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gradient_against_differences(tbn, act):
    # central differences of the 64-bit block: their own error is |act'''| step^2 / 6 and 2^-52 / step, below 1e-6 here
    gu = torch.randn(6, 2 * 40, generator=torch.Generator().manual_seed(3)).to(BF).cuda()
    gu[:, :40][gu[:, :40].abs() < 0.01] = 0.5  # relu's corner
    dh = torch.randn(6, 40, generator=torch.Generator().manual_seed(4)).to(BF).cuda()
    dgu, _ = tbn.glu_bwd(dh, gu=gu, act=act)
    step = 1e-4
    value = lambda g, u: act64(act, g)[0] * u  # noqa: E731
    g, u = gu.double().chunk(2, 1)
    dg = (value(g + step, u) - value(g - step, u)) / (2 * step) * dh.double()
    du = (value(g, u + step) - value(g, u - step)) / (2 * step) * dh.double()
    want = torch.cat([dg, du], 1)
    assert ((dgu.double() - want).abs() <= H * want.abs() + 1e-5).all()


def test_the_rest_of_the_backward_pass_is_a_layers(tbn):
    """dgu goes on through the calls of a layer of 2 f filters: dx and dW of the block, by autograd in 64 bits."""
    rows, c, f = 96, 64, 40
    x, codes, alpha, dh, w = block(tbn, rows, c, f)
    h, gu = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    dgu, _ = tbn.glu_bwd(dh, x=x, codes=codes, alpha=alpha)
    d = tbn.ConvDesc(rows, 1, 1, c, 2 * f, 1, 1)
    dx = tbn.conv2d_bwd_data(d, dgu, codes, alpha, out_dtype=F).view(rows, c)
    dw = tbn.conv2d_bwd_weight(d, x, dgu).view(2 * f, c)
    x64, w64 = x.double().requires_grad_(), w.clone().requires_grad_()
    p = x64 @ w64.t()
    (torch.nn.functional.silu(p[:, :f]) * p[:, f:] * dh.double()).sum().backward()
    # dgu and alpha rounded to bf16 (H each), the sums' own 2^-23 a term far below
    got = dgu.double().abs()
    assert ((dx.double() - x64.grad).abs() <= (2 * H + 1e-4) * (got @ w.abs()) + 1e-6).all()
    assert ((dw.double() - w64.grad).abs() <= (H + 1e-4) * (got.t() @ x.double().abs()) + 1e-6).all()


@pytest.mark.parametrize("rows,c,f", [(3, 40, 20), (3, 20000, 20), (16, 100, 50), (50, 300, 70), (70, 100, 40), (1000, 100, 2000), (4100, 72, 1601)])
def test_what_is_not_finite_stays_in_its_row(tbn, rows, c, f):
    x, codes, alpha, dh, w = block(tbn, rows, c, f)
    clean = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    bad = rows // 2
    for v in (float("nan"), float("inf")):
        y = x.clone()
        y[bad, c - 1] = v
        got = tbn.glu_fwd(y, codes, alpha, want_gu=True)
        back, _ = tbn.glu_bwd(dh, x=y, codes=codes, alpha=alpha)
        keep = torch.arange(rows, device="cuda") != bad
        for a, b in zip(got, clean):
            assert torch.equal(a[keep], b[keep])
        assert torch.isfinite(back[keep]).all()
        assert not torch.isfinite(got[1][bad]).any()


def test_large_gates(tbn):
    # exponentials that overflow or vanish: act(g) goes to g or 0, its slope to 1 or 0
    gu = torch.tensor([[-300.0, -100.0, -60.0, 60.0, 100.0, 300.0, 3e38, -3e38] + [1.0] * 8], device="cuda").to(BF)
    dh = torch.ones(1, 8, device="cuda", dtype=BF)
    for act in ("silu", "gelu", "relu"):
        dgu, h = tbn.glu_bwd(dh, gu=gu, act=act, want_h=True, out_dtype=F)
        big = gu[0, :8].float()
        want = big.clamp(min=0)
        assert torch.isfinite(h).all() and torch.isfinite(dgu).all()
        assert ((h[0] - want).abs() <= 1e-6 * want + 1e-20).all()
        assert torch.equal(dgu[0, :8].float(), (big > 0).float()) or (dgu[0, :8].float() - (big > 0).float()).abs().max() < 1e-20


def test_shapes_views_and_caller_outputs(tbn):
    x, codes, alpha, dh, w = block(tbn, 12, 48, 24)
    h0, gu0 = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    h, gu = tbn.glu_fwd(x.view(3, 2, 2, 48), codes, alpha, want_gu=True)
    assert h.shape == (3, 2, 2, 24) and gu.shape == (3, 2, 2, 48) and torch.equal(h.view_as(h0), h0) and torch.equal(gu.view_as(gu0), gu0)
    out = torch.full((12, 24), 7.0, device="cuda")
    assert tbn.glu_fwd(x, codes, alpha, h=out)[0] is out and torch.equal(out, tbn.glu_fwd(x, codes, alpha, out_dtype=F)[0])
    dgu = torch.zeros(12, 48, dtype=BF, device="cuda")
    assert tbn.glu_bwd(dh, gu=gu0, dgu=dgu)[0] is dgu and torch.equal(dgu, tbn.glu_bwd(dh, gu=gu0)[0])
    # outputs between rows of guards: nothing else is written
    for rows, c, f in ((3, 40, 21), (40, 300, 37), (70, 100, 41), (1000, 72, 2001)):
        x, codes, alpha, dh, w = block(tbn, rows, c, f)
        flat = torch.full((rows * f + 64,), 3.0, device="cuda")
        at = flat[32:32 + rows * f].view(rows, f)
        tbn.glu_fwd(x, codes, alpha, h=at)
        assert (flat[:32] == 3).all() and (flat[-32:] == 3).all()
        assert torch.equal(at, tbn.glu_fwd(x, codes, alpha, out_dtype=F)[0])
    with pytest.raises(ValueError, match="contiguous"):
        tbn.glu_fwd(x.t(), tbn.quantize(torch.randn(8, 1000, device="cuda"))[0], alpha[:8])


@pytest.mark.parametrize("rows,c,f", [(2, 512, 300), (16, 1000, 300), (100, 2000, 300), (300, 513, 4500), (1000, 130, 2000), (4100, 72, 1600)])
def test_same_bits_from_call_to_call(tbn, rows, c, f):
    x, codes, alpha, dh, w = block(tbn, rows, c, f)
    first = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(first, tbn.glu_fwd(x, codes, alpha, want_gu=True)))


def test_more_than_2_31_values(tbn):
    """Projections of 2^31 values and more: rows from either end and around the border against those rows alone."""
    rows, c, f = (1 << 20) + 77, 64, 1032
    w = torch.randn(2 * f, c, device="cuda")
    codes, alpha, _ = tbn.quantize(w)
    x = torch.randn(rows, c, device="cuda").to(BF)
    h, gu = tbn.glu_fwd(x, codes, alpha, want_gu=True)
    assert gu.numel() > 1 << 31
    values = torch.where(w > 0, 1.0, -1.0).double() * torch.where(w.abs() > 1, 2.0, 1.0) * alpha.double()[:, None]
    at = torch.cat([torch.arange(40), (1 << 31) // (2 * f) + torch.arange(-20, 20), rows - 1 - torch.arange(40)]).cuda()
    gu64, e, h64, eh, _, _ = expect(x[at], values, "silu")
    check(gu[at], gu64, e, "gu")
    check(h[at], h64, eh, "h")
    dh = torch.randn(rows, f, device="cuda").to(BF)
    dgu, _ = tbn.glu_bwd(dh, gu=gu)
    _, _, _, _, want, err = expect(x[at], values, "silu", dh[at], gu=gu[at])
    check(dgu[at], want, err, "dgu")
