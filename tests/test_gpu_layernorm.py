"""Layer normalisation against the definition in 64 bits, for every kernel (teams of 8 lanes to 1024 threads, rows
beyond the registers), odd and short rows, both types on either side.

Tolerances, from u = 2^-24: a sum of c values is c / (8 T) * 8 serial additions in a thread and a tree over T of them,
below 64 roundings for c up to 65536 (n = 64 here), so mean is off by at most n u mean|x|; x - mean adds one rounding
and the scaling a few more, each of the value's size.  The rounding to the output's type comes on top (half a step).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
BF, F = torch.bfloat16, torch.float32

# one row length or two of each kernel, and its borders: 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768
SIZES = [(1, 1), (1, 512), (5, 7), (3, 8), (2, 63), (70, 64), (33, 100), (9, 200), (4, 256), (5, 257), (6, 512), (130, 1000),
         (3, 1031), (7, 2048), (2, 3136), (5, 4096), (3, 8192), (2, 8200), (1, 16384), (2, 20001), (2, 32768), (3, 40003)]


def make(rows, c, xt, yt, seed, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, c, generator=g) * 1.5 + mean).to(xt)
    dy = torch.randn(rows, c, generator=g).to(yt)
    return x, dy, 1 + 0.2 * torch.randn(c, generator=g), 0.1 * torch.randn(c, generator=g)


def check(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol
    assert not torch.isnan(off).any() and off.max() <= 0, "%s: %g over the tolerance" % (what, off.max())


def reference(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    s = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mean) * s
    return xh * (1 if gamma is None else gamma.double()) + (0 if beta is None else beta.double()), mean, s, xh


def check_forward(x, gamma, beta, eps, y, mean, inv_std):
    want, mu, s, xh = reference(x, gamma, beta, eps)
    size = x.double().abs().mean(1, keepdim=True)
    tm = 64 * U * size
    check(mean, mu[:, 0], tm[:, 0], "mean")
    # the variance moves by 2 tm |x - mean| on average (xh has mean square 1 at most) and by its own sum's roundings
    ts = s * (2 * tm * s + 80 * U)
    check(inv_std, s[:, 0], ts[:, 0], "inv_std")
    g = 1 if gamma is None else gamma.double().abs()
    b = 0 if beta is None else beta.double().abs()
    tol = g * (tm * s + (x.double() - mu).abs() * ts + 6 * U * xh.abs()) + U * b + HALF[y.dtype] * want.abs()
    check(y, want, tol * 1.001, "y")


@pytest.mark.parametrize("rows,c", SIZES)
@pytest.mark.parametrize("xt,yt", [(BF, BF), (F, BF), (BF, F), (F, F)])
def test_forward(tbn, rows, c, xt, yt):
    x, _, gamma, beta = make(rows, c, xt, yt, c)
    y, mean, inv_std = tbn.layernorm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), out_dtype=yt)
    assert y.dtype == yt and y.shape == x.shape
    check_forward(x, gamma, beta, 1e-5, y, mean, inv_std)


@pytest.mark.parametrize("rows,c", SIZES)
@pytest.mark.parametrize("xt,yt", [(BF, BF), (F, BF), (BF, F), (F, F)])
def test_backward(tbn, rows, c, xt, yt):
    x, dy, gamma, _ = make(rows, c, xt, yt, c + 1)
    _, mean, s, _ = reference(x, None, None, 1e-5)
    mean, s = mean.float(), s.float()
    dx, dgamma, dbeta = tbn.layernorm_bwd(x.cuda(), dy.cuda(), mean[:, 0].cuda(), s[:, 0].cuda(), gamma.cuda())
    check_backward(x, dy, mean.double(), s.double(), gamma.double(), dx, dgamma, dbeta)


@pytest.mark.parametrize("rows,c", [(37, 16385), (75, 18432), (9, 40003), (4, 65536), (1030, 16392)])
@pytest.mark.parametrize("xt,yt", [(BF, BF), (F, BF), (BF, F), (F, F)])
def test_backward_long(tbn, rows, c, xt, yt):
    # several rows a share, shares that end early, columns that end inside a block
    test_backward(tbn, rows, c, xt, yt)


def check_backward(x, dy, mean, s, gamma, dx, dgamma, dbeta):
    c = x.shape[1]
    xh, d = (x.double() - mean) * s, dy.double()
    h = d * gamma
    want = s * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    # each term is rounded a few times, the means by 64 roundings of what is added
    m1, m2 = h.abs().mean(1, keepdim=True), (h * xh).abs().mean(1, keepdim=True)
    tol = s * U * (6 * h.abs() + 70 * m1 + 80 * xh.abs() * m2) + HALF[dx.dtype] * want.abs()
    check(dx, want, tol * 1.001, "dx")
    n = 40 + x.shape[0] / 512  # rows in turn in a team, the teams of a block, the blocks
    check(dgamma, (d * xh).sum(0), n * U * (d * xh).abs().sum(0) + 1e-300, "dgamma")
    check(dbeta, d.sum(0), n * U * d.abs().sum(0) + 1e-300, "dbeta")
    assert dgamma.shape == dbeta.shape == (c,)


@pytest.mark.parametrize("rows,c", [(4099, 96), (3000, 777), (1500, 2500)])
def test_many_rows(tbn, rows, c):
    # more rows than teams at once: every team walks several
    x, dy, gamma, beta = make(rows, c, BF, BF, 5)
    y, mean, inv_std = tbn.layernorm_fwd(x.cuda(), gamma.cuda(), beta.cuda())
    check_forward(x, gamma, beta, 1e-5, y, mean, inv_std)
    out = tbn.layernorm_bwd(x.cuda(), dy.cuda(), mean, inv_std, gamma.cuda())
    check_backward(x, dy, mean.cpu().double()[:, None], inv_std.cpu().double()[:, None], gamma.double(), *out)
    again = tbn.layernorm_bwd(x.cuda(), dy.cuda(), mean, inv_std, gamma.cuda())
    assert all(torch.equal(p, q) for p, q in zip(out, again))


def test_without_parameters_and_statistics(tbn):
    x, dy, _, _ = make(6, 300, F, F, 2)
    y, mean, inv_std = tbn.layernorm_fwd(x.cuda(), want_stats=False)
    assert mean is None and inv_std is None
    z, mean, inv_std = tbn.layernorm_fwd(x.cuda())
    assert torch.equal(y, z)
    check_forward(x, None, None, 1e-5, y, mean, inv_std)
    out = tbn.layernorm_bwd(x.cuda(), dy.cuda(), mean, inv_std)
    check_backward(x, dy, mean.cpu().double()[:, None], inv_std.cpu().double()[:, None], torch.ones(300).double(), *out)


def test_far_mean_and_constant_rows(tbn):
    # the centred sum of squares is taken about the mean: no cancellation where the mean is large
    x, _, gamma, beta = make(8, 1000, F, F, 3, mean=1000.0)
    x[3] = 7.0  # constant: y = beta
    y, mean, inv_std = tbn.layernorm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), eps=1e-3)
    check_forward(x, gamma, beta, 1e-3, y, mean, inv_std)


def test_rows_do_not_mix(tbn):
    # NaN and infinities stay in their rows (and, backward, in the sums over rows)
    x, dy, gamma, beta = make(40, 72, BF, BF, 4)
    clean = tbn.layernorm_fwd(x.cuda(), gamma.cuda(), beta.cuda())
    x2 = x.clone()
    x2[5, 3], x2[17, 71], x2[30] = float("nan"), float("inf"), float("-inf")
    dirty = tbn.layernorm_fwd(x2.cuda(), gamma.cuda(), beta.cuda())
    keep = [i for i in range(40) if i not in (5, 17, 30)]
    for p, q in zip(clean, dirty):
        assert torch.equal(p[keep], q[keep])
    assert torch.isnan(dirty[0][[5, 17, 30]].float()).all()
    dx = tbn.layernorm_bwd(x.cuda(), dy.cuda(), clean[1], clean[2], gamma.cuda())[0]
    dx2 = tbn.layernorm_bwd(x2.cuda(), dy.cuda(), dirty[1], dirty[2], gamma.cuda())[0]
    assert torch.equal(dx[keep], dx2[keep])


def test_gradient_by_differences(tbn):
    # dx, dgamma, dbeta of sum(y w) against central differences of the kernel's own fp32 forward pass: with step h
    # the difference is off by rounding, 2^-22 |terms| / h, and by h^2 times the third derivative (of order 1 here)
    x, w, gamma, beta = (t.cuda() for t in make(2, 24, F, F, 9))
    _, mean, inv_std = tbn.layernorm_fwd(x, gamma, beta)
    grads = tbn.layernorm_bwd(x, w, mean, inv_std, gamma)
    h = 2.0 ** -6

    def value(*p):
        return float((tbn.layernorm_fwd(*p)[0].double() * w.double()).sum())

    for k, (p, g) in enumerate(zip((x, gamma, beta), grads)):
        for i in range(0, p.numel(), 5):
            args = [t.clone() for t in (x, gamma, beta)]
            args[k].view(-1)[i] += h
            up = value(*args)
            args[k].view(-1)[i] -= 2 * h
            assert abs((up - value(*args)) / (2 * h) - float(g.reshape(-1)[i])) < 2e-3


def test_outputs_given_and_other_stream(tbn):
    x, dy, gamma, beta = (t.cuda() for t in make(50, 520, BF, BF, 6))
    torch.cuda.synchronize()
    want = tbn.layernorm_fwd(x, gamma, beta)
    wanted = tbn.layernorm_bwd(x, dy, want[1], want[2], gamma)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    flat = torch.full((1041,), 7.0, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = tbn.layernorm_fwd(x, gamma, beta)
        # views at the alignment of an element
        out = tbn.layernorm_bwd(x, dy, got[1], got[2], gamma, dgamma=flat[1:521], dbeta=flat[521:])
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got)) and all(torch.equal(p, q) for p, q in zip(wanted, out))
    assert flat[0] == 7.0 and torch.equal(flat[1:521], wanted[1])


def test_captured(tbn):
    x, dy, gamma, beta = (t.cuda() for t in make(600, 130, BF, BF, 7))

    def step():
        y, mean, inv_std = tbn.layernorm_fwd(x, gamma, beta)
        return (y,) + tbn.layernorm_bwd(x, dy, mean, inv_std, gamma)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2, 3):
        x.copy_(make(600, 130, BF, BF, seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))
