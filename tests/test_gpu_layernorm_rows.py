"""Layer normalisation whose teams walk over several rows, against the formulas in 64 bits: more rows than the largest grids hold at
once (test_many_rows of test_gpu_layernorm.py gives each team of the forward pass one), random values in each, so that a row that
was taken for its neighbour shows.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U, EPS = 2.0 ** -24, 1e-5
BF, F = torch.bfloat16, torch.float32
HALF = {F: U, BF: 2.0 ** -8}

# one team of the forward and backward passes after the other (8, 16, 32, 64 lanes; 2 and 4 pieces; blocks), whole and odd rows;
# the last ones: rows that are read again, forward (more than 512 of them), backward (more than 4096) and in shares of many rows
WALKS = [(70000, 40, BF, BF), (70001, 39, F, BF), (33000, 100, BF, F), (33003, 128, F, F), (17000, 200, BF, BF), (17001, 255, F, F),
         (9000, 500, BF, BF), (9001, 504, F, BF), (9000, 1000, F, F), (9001, 1023, BF, BF), (9000, 1500, BF, F), (9001, 2048, F, BF),
         (2500, 3000, BF, BF), (2501, 4095, F, F), (2500, 8000, F, BF), (2501, 6001, BF, BF), (1100, 16384, BF, BF), (1101, 9999, F, F),
         (1100, 32768, BF, BF), (600, 20001, F, BF), (4200, 16392, BF, BF)]


def close(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert not torch.isnan(off).any() and off.max() <= 0, "%s: %g over the tolerance" % (what, off.max())


@pytest.mark.parametrize("rows,c,xt,yt", WALKS, ids=lambda v: str(v).split(".")[-1])
def test_layer_norm_teams_of_several_rows(tbn, rows, c, xt, yt):
    # Tolerances: sums of c values as in test_gpu_layernorm.py (64 roundings up to c = 65536).  The sums over rows: at most rows / 256
    # in turn in a team (the smallest grid), 32 teams of a block, 512 / 32 blocks in turn, 32 of those and three roundings of xh,
    # below 90 + rows / 256.  The reference is the formula in 64 bits, on the GPU
    g = torch.Generator(device="cuda").manual_seed(rows + c)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    x, dy = (normal(rows, c) * 1.5 + 0.3).to(xt), normal(rows, c).to(yt)
    gamma, beta = 1 + 0.2 * normal(c), 0.1 * normal(c)
    y, mean, inv_std = tbn.layernorm_fwd(x, gamma, beta, eps=EPS, out_dtype=yt)
    xd = x.double()
    mu = xd.mean(1, keepdim=True)
    s = 1 / ((xd - mu).square().mean(1, keepdim=True) + EPS).sqrt()
    t_mu = 64 * U * xd.abs().mean(1, keepdim=True)
    t_s = s * (2 * t_mu * s + 80 * U)
    close(mean, mu[:, 0], t_mu[:, 0], "mean")
    close(inv_std, s[:, 0], t_s[:, 0], "inv_std")
    xh = (xd - mu) * s
    want = xh * gamma + beta
    tol = gamma.abs() * (t_mu * s + (xd - mu).abs() * t_s + 6 * U * xh.abs()) + U * beta.abs() + HALF[yt] * want.abs()
    close(y, want, tol * 1.001, "y")
    del y, want, tol

    dx, dgamma, dbeta = tbn.layernorm_bwd(x, dy, mean, inv_std, gamma)
    mu, s = mean.double()[:, None], inv_std.double()[:, None]
    xh, d = (xd - mu) * s, dy.double()
    del xd
    n = (90 + rows / 256) * U
    close(dgamma, (d * xh).sum(0), n * (d * xh).abs().sum(0), "dgamma")
    close(dbeta, d.sum(0), n * d.abs().sum(0), "dbeta")
    h = d * gamma
    want = s * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    m1, m2 = h.abs().mean(1, keepdim=True), (h * xh).abs().mean(1, keepdim=True)
    close(dx, want, s * U * (6 * h.abs() + 70 * m1 + 80 * xh.abs() * m2) * 1.001 + HALF[xt] * want.abs() * 1.001, "dx")


@pytest.mark.parametrize("rows,c,xt,yt", [(1, 65537, F, F), (2, (1 << 20) + 8, BF, BF), (1, 3000001, F, BF)],
                         ids=lambda v: str(v).split(".")[-1])
def test_layer_norm_of_very_long_rows(tbn, rows, c, xt, yt):
    # a thread of 1024 adds c / 1024 values in turn, a tree of 10 and 16 waves follow: n roundings of a sum of c values; its share
    # of the variance is twice the mean's error and n of its own
    n = (c / 1024 + 8 + 26) * U
    g = torch.Generator(device="cuda").manual_seed(c)
    x, dy = (torch.randn(rows, c, generator=g, device="cuda") + 0.3).to(xt), torch.randn(rows, c, generator=g, device="cuda").to(yt)
    gamma = 1 + 0.2 * torch.randn(c, generator=g, device="cuda")
    y, mean, inv_std = tbn.layernorm_fwd(x, gamma, out_dtype=yt)
    xd, d = x.double(), dy.double()
    mu = xd.mean(1, keepdim=True)
    s = 1 / ((xd - mu).square().mean(1, keepdim=True) + EPS).sqrt()
    t_mu = n * xd.abs().mean(1, keepdim=True)
    t_s = s * (2 * t_mu * s + n + 8 * U)
    close(mean, mu[:, 0], t_mu[:, 0], "mean")
    close(inv_std, s[:, 0], t_s[:, 0], "inv_std")
    xh = (xd - mu) * s
    want = xh * gamma
    close(y, want, gamma.abs() * (t_mu * s + (xd - mu).abs() * t_s + 6 * U * xh.abs()) * 1.001 + HALF[yt] * want.abs() * 1.001, "y")
    dx, dgamma, dbeta = tbn.layernorm_bwd(x, dy, mean, inv_std, gamma)
    mu, s = mean.double()[:, None], inv_std.double()[:, None]
    xh, h = (xd - mu) * s, d * gamma
    close(dgamma, (d * xh).sum(0), 8 * U * (d * xh).abs().sum(0), "dgamma")
    close(dbeta, d.sum(0), 2 * U * d.abs().sum(0), "dbeta")
    want = s * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    m1, m2 = h.abs().mean(1, keepdim=True), (h * xh).abs().mean(1, keepdim=True)
    tol = s * (6 * U * h.abs() + (n + 4 * U) * m1 + (n + 12 * U) * xh.abs() * m2)
    close(dx, want, tol * 1.001 + HALF[xt] * want.abs() * 1.001, "dx")
