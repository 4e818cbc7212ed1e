"""Rows in 8-bit integers and their products against the definitions: the integers and scales bit for bit, the sums exactly, in 64 bits.

Tolerances: the sum is rounded to fp32 once, both scales' product (and a further factor) once each, the product with the sum, the bias and
the residual once each: 2^-24 of its value every time.  bf16 adds 2^-8 of the result, half a step.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F, I8 = torch.bfloat16, torch.float32, torch.int8


def rows_reference(x):
    """On the CPU in fp32, where each operation is rounded by itself."""
    x = x.float().cpu()
    finite = torch.where(torch.isfinite(x), x.abs(), torch.zeros(()))
    t = finite.amax(1)
    some = t >= 2.0 ** -100
    inv = torch.where(some, torch.div(torch.full_like(t, 127.0), torch.where(some, t, torch.ones_like(t))), torch.zeros_like(t))
    q = torch.nan_to_num((x * inv[:, None]).round().clamp(-127, 127), nan=0.0)
    q[~some] = 0
    q[torch.isnan(x)] = 0
    pad = -(-x.shape[1] // 16) * 16
    out = torch.zeros(x.shape[0], pad, dtype=I8)
    out[:, :x.shape[1]] = q.to(I8)
    return out, torch.where(some, t * torch.tensor(1 / 127, dtype=F), torch.zeros_like(t))


@pytest.mark.parametrize("rows,c", [(1, 1), (3, 7), (5, 16), (4, 17), (2, 127), (9, 1000), (6, 1024), (7, 1025), (3, 4096), (5, 4100), (2, 8192),
                                    (3, 8200), (2, 40001), (1000, 72), (1, 131056)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_rows(tbn, rows, c, dtype):
    g = torch.Generator().manual_seed(rows * 1009 + c)
    x = (torch.randn(rows, c, generator=g) * torch.rand(rows, 1, generator=g) * 10).to(dtype)
    q, scale = tbn.quantize_rows_i8(x.cuda())
    want_q, want_s = rows_reference(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(scale.cpu(), want_s)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("c", [40, 1500, 9000])
def test_rows_that_are_not_ordinary(tbn, c, dtype):
    nan, inf = float("nan"), float("inf")
    x = torch.randn(10, c, generator=torch.Generator().manual_seed(c))
    x[0] = 0.0
    x[1, ::3] = nan
    x[2, 5], x[2, 6] = inf, -inf
    x[3] = nan
    x[4] = inf
    x[5] = x[5] * 2.0 ** -101  # below the smallest row that has a scale, or near it
    x[6] = 2.0 ** -100
    x[7] = x[7].clamp(-3, 3) * 1e38
    x[8] = -0.0
    x[9, 0] = 1e30
    x = x.to(dtype)
    q, scale = tbn.quantize_rows_i8(x.cuda())
    want_q, want_s = rows_reference(x)
    assert torch.equal(scale.cpu(), want_s)
    assert torch.equal(q.cpu(), want_q)
    assert q[2, 5] == 127 and q[2, 6] == -127 and not q[3].any() and not q[4].any() and scale[4] == 0


def test_ties_go_to_the_even_integer(tbn):
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -126.5]], device="cuda")
    q, scale = tbn.quantize_rows_i8(x)
    assert q[0, :8].tolist() == [127, 0, 2, 2, 0, -2, 126, -126] and scale.item() == pytest.approx(1.0)


def product_case(rows, n, c, seed=0):
    g = torch.Generator().manual_seed(seed * 7 + rows * 31 + n * 17 + c)
    q = torch.randint(-128, 128, (rows, c), generator=g, dtype=torch.int16).to(I8)
    w = torch.randint(-128, 128, (n, c), generator=g, dtype=torch.int16).to(I8)
    return q.cuda(), (torch.rand(rows, generator=g) + 0.01).cuda(), w.cuda(), (torch.rand(n, generator=g) * 0.1).cuda(), g


def check(y, acc, s, bias=0.0, res=0.0, relu=False):
    want = acc * s + bias + res
    mags = (acc * s).abs() + (bias.abs() if isinstance(bias, torch.Tensor) else 0) + (res.abs() if isinstance(res, torch.Tensor) else 0)
    err = 6 * 2.0 ** -24 * mags
    if relu:
        want = want.clamp(min=0)
    rounding = 2.0 ** -8 if y.dtype == BF else 2.0 ** -24
    assert y.shape == want.shape
    off = (y.double() - want).abs() - err - rounding * (want.abs() + err) - 1e-38
    assert off.max().item() <= 0, off.max().item()


SHAPES = [(1, 1, 16), (1, 5, 32), (2, 33, 16), (16, 100, 48), (7, 1000, 1008), (16, 16400, 80), (1, 16385, 144), (4, 70000, 272),  # few rows
          (16, 300, 4096), (5, 18000, 2064), (16, 50, 4112), (9, 9001, 8192),                         # ... all of a block's waves
          (3, 64, 131056), (16, 33, 8208), (1, 1000, 8208),                                           # ... x with the weights
          (17, 1, 16), (17, 40, 128), (64, 64, 512), (33, 257, 144), (17, 300, 1008), (777, 2049, 144), (320, 3500, 560),  # 64 x 64
          (17, 300, 2064), (100, 500, 4112), (200, 130, 4112), (64, 1000, 2048), (40, 64, 131056),    # ... in groups of waves
          (1000, 2100, 176), (1100, 1900, 304),                                                       # 128 x 64
          (1700, 1700, 176), (1290, 2048, 1008),                                                      # 128 x 128 by eight waves
          (2100, 2200, 176), (1500, 2900, 1008),                                                      # ... by four
          (3100, 4100, 304), (4000, 3333, 128)]                                                       # 256 x 256


@pytest.mark.parametrize("rows,n,c", SHAPES)
def test_product(tbn, rows, n, c):
    q, xs, w, ws, g = product_case(rows, n, c)
    acc = q.double() @ w.double().t()  # exact: below 2^53
    s = xs.double()[:, None] * ws.double()
    check(tbn.matmul_i8(q, xs, w, ws, out_dtype=F), acc, s)
    check(tbn.matmul_i8(q, xs, w, ws), acc, s)
    bias, factor = torch.randn(n, generator=g).cuda() * 100, torch.randn(n, generator=g).cuda()
    for dtype in (F, BF):
        res = (torch.randn(rows, n, generator=g) * 100).to(dtype).cuda()
        y = tbn.matmul_i8(q, xs, w, ws, scale=factor, bias=bias, residual=res, relu=True, out_dtype=dtype)
        check(y, acc, s * factor.double(), bias.double(), res.double(), True)
        into = res.clone()
        assert tbn.matmul_i8(q, xs, w, ws, scale=factor, bias=bias, residual=into, relu=True, y=into) is into
        assert torch.equal(into, y)


def test_sums_up_to_the_largest(tbn):
    c = 131056
    for rows in (1, 17, 40):
        q = torch.full((rows, c), -128, dtype=I8, device="cuda")
        w = torch.stack([torch.full((c,), v, dtype=I8, device="cuda") for v in (-128, 127, 1)])
        y = tbn.matmul_i8(q, torch.ones(rows, device="cuda"), w, torch.ones(3, device="cuda"), out_dtype=F)
        assert torch.equal(y[-1].cpu(), torch.tensor([128.0 * 128 * c, -128.0 * 127 * c, -128.0 * c]).float())


def test_scales_that_are_not_finite_stay_in_their_row_and_channel(tbn):
    for rows, n, c in ((5, 40, 64), (50, 70, 1008), (1000, 2100, 64)):
        q, xs, w, ws, _ = product_case(rows, n, c)
        clean = tbn.matmul_i8(q, xs, w, ws, out_dtype=F)
        xs[rows // 2], ws[n // 3] = float("nan"), float("inf")
        y = tbn.matmul_i8(q, xs, w, ws, relu=True, out_dtype=F)
        keep_r, keep_n = torch.arange(rows) != rows // 2, torch.arange(n) != n // 3
        assert torch.equal(y[keep_r.cuda()][:, keep_n.cuda()], clean[keep_r.cuda()][:, keep_n.cuda()].clamp(min=0))
        assert torch.isnan(y[rows // 2]).all()


def test_a_layer_in_8_bits(tbn):
    """Weights and activations through both calls: off from the real layer by half a step of either's rounding, and no more."""
    g = torch.Generator().manual_seed(5)
    for rows in (1, 30, 300):
        x, w = torch.randn(rows, 500, generator=g).cuda(), torch.randn(70, 500, generator=g).cuda()
        q, xs = tbn.quantize_rows_i8(x)
        wq, ws = tbn.quantize_rows_i8(w)
        y = tbn.matmul_i8(q, xs, wq, ws, out_dtype=F).double()
        x64, w64 = x.double(), w.double()
        # |x - s q| <= s / 2 (1 + 2^-20), likewise w
        ex, ew = xs.double()[:, None] * 0.5001, ws.double()[:, None] * 0.5001
        bound = ex * w64.abs().sum(1) + (x64.abs() + ex).sum(1, keepdim=True) * ew.t()
        assert ((y - x64 @ w64.t()).abs() <= bound).all()


def test_guards_and_caller_outputs(tbn):
    for rows, n, c in ((3, 21, 32), (40, 37, 1008), (70, 41, 64), (1000, 2101, 64)):
        q, xs, w, ws, _ = product_case(rows, n, c)
        flat = torch.full((rows * n + 64,), 3.0, device="cuda")
        at = flat[32:32 + rows * n].view(rows, n)
        assert tbn.matmul_i8(q, xs, w, ws, y=at) is at
        assert (flat[:32] == 3).all() and (flat[-32:] == 3).all() and torch.equal(at, tbn.matmul_i8(q, xs, w, ws, out_dtype=F))
    x = torch.randn(2, 3, 40, device="cuda")
    q, s = torch.full((6, 48), 9, dtype=I8, device="cuda"), torch.zeros(6, device="cuda")
    a, b = tbn.quantize_rows_i8(x, q=q, scale=s)
    assert a is q and b is s and not q[:, 40:].any()
    assert all(torch.equal(u, v) for u, v in zip((q, s), tbn.quantize_rows_i8(x)))


def test_more_than_2_31_values(tbn):
    rows, c = (1 << 21) + 5, 1030
    x = torch.empty(rows, c, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    q, s = tbn.quantize_rows_i8(x)
    at = torch.cat([torch.arange(9), (1 << 31) // c + torch.arange(-4, 4), rows - 1 - torch.arange(9)]).cuda()
    want_q, want_s = rows_reference(x[at])
    assert torch.equal(q[at].cpu(), want_q) and torch.equal(s[at].cpu(), want_s)
    del x, q
    rows, n, c = 70001, 32768, 32
    q, xs, w, ws, _ = product_case(rows, n, c)
    y = tbn.matmul_i8(q, xs, w, ws)
    at = torch.cat([torch.arange(9), (1 << 31) // n + torch.arange(-4, 4), rows - 1 - torch.arange(9)]).cuda()
    check(y[at], q[at].double() @ w.double().t(), xs[at].double()[:, None] * ws.double())
