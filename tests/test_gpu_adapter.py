"""Low-rank adapters against the formulas in 64 bits: ranks from 1 to 128, few rows with adapters of their own and long
batches, odd sizes, rows without an adapter, every type.

Tolerances, from u = 2^-24: products of bf16 factors are exact, a sum of n of them in fp32 is off by at most
(n / 32 + 64) u times the sum of the magnitudes (an MFMA adds 32 in at most 8 roundings counted as one each; waves, splits and
adapters behind them).  A factor of 32 bits enters exactly, as three bf16 numbers each 2^-8 of the one before (half a step
of bf16): a product of two such factors leaves out mid lo, lo mid and lo lo, 2 * 2^-24 + 2^-32 of it, and three or six
terms are added where there was one.  The rounding to the output's type comes on top (half a step).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U, SPLIT = 2.0 ** -24, 8 * 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
BF, F = torch.bfloat16, torch.float32


def make(rows, c, k, rank, bank, wt=BF, xt=BF, ot=BF, index=None, seed=0):
    g = torch.Generator().manual_seed(seed + rows + c)

    def normal(*shape):
        return torch.randn(*shape, generator=g)

    if index is None:  # runs of rows, some without an adapter
        index = torch.repeat_interleave(torch.randint(-1, bank, (rows,), generator=g), torch.randint(1, 9, (rows,), generator=g))[:rows]
    return {"x": normal(rows, c).to(xt), "dy": normal(rows, k).to(xt), "index": index.to(torch.int32),
            "a": (normal(bank, rank, c) * c ** -0.5).to(wt), "b": normal(bank, k, rank).to(wt),
            "scale": normal(bank).abs() + 0.1, "res_y": normal(rows, k).to(ot), "res_x": normal(rows, c).to(ot)}


def check(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol
    assert not torch.isnan(off).any() and off.max() <= 0, "%s: %g over the tolerance" % (what, off.max())


def own(s):
    """[rows] adapter of each row and whether it has one."""
    i = s["index"].long()
    has = (i >= 0) & (i < s["a"].shape[0])
    return torch.where(has, i, 0), has.double()[:, None]


def check_forward(s, y, t, residual=True, scaled=True):
    i, has = own(s)
    x, a, b = s["x"].double(), s["a"].double(), s["b"].double()
    scale = (s["scale"].double() if scaled else torch.ones(a.shape[0]).double())[i][:, None]
    want_t = torch.stack([x[r] @ a[i[r]].t() for r in range(len(i))]) * has
    size_t = torch.stack([x[r].abs() @ a[i[r]].abs().t() for r in range(len(i))]) * has
    f32 = s["x"].dtype == F or s["a"].dtype == F
    tol_t = ((x.shape[1] / 32 + 64) * U + (SPLIT if f32 else 0)) * size_t
    if t is not None:
        check(t, want_t, tol_t + 1e-300, "t")
    delta = torch.stack([b[i[r]] @ want_t[r] for r in range(len(i))]) * scale * has
    size = torch.stack([b[i[r]].abs() @ (want_t[r].abs() * (SPLIT + 70 * U) + tol_t[r]) for r in range(len(i))]) * scale * has
    want = delta + (s["res_y"].double() if residual else 0)
    check(y, want, size + 2 * U * want.abs() + HALF[y.dtype] * want.abs(), "y")


def check_backward(s, t, dx, da, db, residual=True, scaled=True):
    i, has = own(s)
    x, dy, a, b, t = s["x"].double(), s["dy"].double(), s["a"].double(), s["b"].double(), t.double().cpu()
    bank, rank = a.shape[:2]
    scale = (s["scale"].double() if scaled else torch.ones(bank).double())[i][:, None]
    n = x.shape[0]
    dt = torch.stack([dy[r] @ b[i[r]] for r in range(n)]) * scale * has
    f32 = s["x"].dtype == F or s["a"].dtype == F
    tol_dt = ((dy.shape[1] / 32 + 64) * U + (SPLIT if f32 else 0)) * torch.stack([dy[r].abs() @ b[i[r]].abs() for r in range(n)]) * scale * has
    if dx is not None:
        want = torch.stack([dt[r] @ a[i[r]] for r in range(n)]) + (s["res_x"].double() if residual else 0)
        size = torch.stack([(dt[r].abs() * (SPLIT + 70 * U) + tol_dt[r]) @ a[i[r]].abs() for r in range(n)])
        check(dx, want, size + 2 * U * want.abs() + HALF[dx.dtype] * want.abs(), "dx")
    mine = torch.nn.functional.one_hot(i, bank).double() * has  # [rows][bank]
    add = (n / 32 + 64) * U + SPLIT
    want = torch.einsum("nb,nr,nc->brc", mine, dt, x)
    check(da, want, torch.einsum("nb,nr,nc->brc", mine, dt.abs() * add + tol_dt, x.abs()) + 1e-300, "da")
    ts = t * scale
    want = torch.einsum("nb,nk,nr->bkr", mine, dy, ts)
    check(db, want, torch.einsum("nb,nk,nr->bkr", mine, dy.abs(), ts.abs() * (add + U)) + 1e-300, "db")


def gpu(s):
    return {k: v.cuda() for k, v in s.items()}


def run(tbn, s, residual=True, scaled=True):
    d = gpu(s)
    scale = d["scale"] if scaled else None
    y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=scale, residual=d["res_y"] if residual else None,
                           out_dtype=s["res_y"].dtype)
    check_forward(s, y, t, residual, scaled)
    out = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=scale,
                          residual=d["res_x"] if residual else None, out_dtype=s["res_x"].dtype)
    check_backward(s, t, *out, residual=residual, scaled=scaled)
    return (y, t) + out


@pytest.mark.parametrize("rank", [1, 3, 8, 16, 17, 32, 40, 64, 100, 128])
@pytest.mark.parametrize("rows", [1, 5, 100])
def test_ranks(tbn, rank, rows):
    run(tbn, make(rows, 200, 136, rank, 3))


@pytest.mark.parametrize("c,k", [(1, 1), (7, 3), (31, 33), (64, 64), (100, 257), (513, 72), (1000, 10), (72, 1001)])
@pytest.mark.parametrize("rows", [2, 79])
def test_sizes(tbn, c, k, rows):
    run(tbn, make(rows, c, k, 5, 2))


@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("xt", [BF, F])
@pytest.mark.parametrize("ot", [BF, F])
@pytest.mark.parametrize("rows,rank", [(3, 8), (90, 20), (70, 70)])
def test_types(tbn, wt, xt, ot, rows, rank):
    run(tbn, make(rows, 168, 90, rank, 4, wt, xt, ot))


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 64, 65, 129])
def test_rows(tbn, rows):
    run(tbn, make(rows, 96, 80, 8, 5))


def test_without_residual_and_scale(tbn):
    run(tbn, make(37, 64, 48, 4, 2), residual=False, scaled=False)


def test_scattered_rows(tbn):
    # every row another adapter than its neighbours, more adapters than a tile has rows
    g = torch.Generator().manual_seed(3)
    for rows in (48, 64, 300):
        run(tbn, make(rows, 128, 96, 16, 40, index=torch.randperm(rows, generator=g) % 40))


def test_rows_without_an_adapter(tbn):
    # none at all, and values outside the bank on either side
    s = make(70, 64, 32, 8, 3, index=torch.full((70,), -1))
    y, t, dx, da, db = run(tbn, s)
    assert torch.equal(y.cpu(), s["res_y"]) and torch.equal(dx.cpu(), s["res_x"])
    assert not t.any() and not da.any() and not db.any()
    odd = torch.tensor([3, -2147483648, 2147483647, 0, -1, 2, 1000, 1] * 9)[:70]
    run(tbn, make(70, 64, 32, 8, 3, index=odd))


def test_adapters_without_rows_get_zero_gradients(tbn):
    s = make(50, 64, 32, 8, 6, index=torch.full((50,), 4))
    _, _, _, da, db = run(tbn, s)
    rest = [0, 1, 2, 3, 5]
    assert not da[rest].any() and not db[rest].any() and da[4].any() and db[4].any()


def test_long_batch(tbn):
    # several lists of rows, several splits, an adapter whose rows lie at both ends
    index = torch.cat([torch.full((4000,), 1), torch.full((1500,), -1), torch.full((3003,), 0), torch.full((700,), 1)])
    s = make(9203, 72, 40, 6, 2, index=index)
    d = gpu(s)
    y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])
    out = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"], residual=d["res_x"])
    check_forward(s, y, t)
    check_backward(s, t, *out)
    again = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"], residual=d["res_x"])
    assert all(torch.equal(p, q) for p, q in zip(out, again))


@pytest.mark.parametrize("rank", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("rows", [3, 33, 130])
def test_whole_columns(tbn, rank, wt, rows):
    # both widths multiples of 256 and ranks of 8: no load has a branch
    run(tbn, make(rows, 512, 768, rank, 3, wt, BF, BF))


@pytest.mark.parametrize("rank", [1, 7, 16, 32, 33, 64, 100, 128])
@pytest.mark.parametrize("bank", [1, 3])
def test_many_rows_of_every_rank(tbn, rank, bank):
    # rows beyond those whose adapters are dealt over blocks; one adapter, and rows taken in the adapters' order
    run(tbn, make(1030, 136, 72, rank, bank))


@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("xt", [BF, F])
@pytest.mark.parametrize("ot", [BF, F])
@pytest.mark.parametrize("rank", [16, 40])
def test_many_rows_of_every_type(tbn, wt, xt, ot, rank):
    run(tbn, make(300, 256, 512, rank, 2, wt, xt, ot))
    run(tbn, make(200, 168, 90, rank, 1, wt, xt, ot))


@pytest.mark.parametrize("c,k", [(1, 1), (7, 3), (100, 257), (513, 72), (512, 1024)])
@pytest.mark.parametrize("rows", [129, 192, 193, 321, 1025])
def test_many_rows_of_every_size(tbn, c, k, rows):
    run(tbn, make(rows, c, k, 5, 2))


@pytest.mark.parametrize("rows", [65, 100, 128])
@pytest.mark.parametrize("c,k,rank", [(512, 1000, 8), (2056, 1032, 20), (72, 3000, 70)])
def test_one_adapter(tbn, rows, c, k, rank):
    # small tiles on the way in, 128 rows at once on the way out
    run(tbn, make(rows, c, k, rank, 1, F, BF, BF))


def test_scattered_long_batches(tbn):
    # every row another adapter than its neighbours, some without one, adapters without rows
    g = torch.Generator().manual_seed(4)
    for rows, bank in ((1100, 17), (700, 2), (200, 1), (2100, 60)):
        index = torch.randint(-2, bank + 2, (rows,), generator=g)
        index[index == bank // 2] = -1
        s = make(rows, 72, 136, 8, bank, index=index)
        _, _, _, da, db = run(tbn, s)
        assert not da[bank // 2].any() and not db[bank // 2].any()


def test_bits_do_not_depend_on_the_neighbours(tbn):
    # a row's results are those of its own values, wherever it lies in the batch and whatever lies beside it
    s = make(1200, 264, 136, 12, 3)
    d = gpu(s)
    y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])
    p = torch.randperm(1200, generator=torch.Generator().manual_seed(1)).cuda()
    y2, t2 = tbn.adapter_fwd(d["x"][p], d["index"][p], d["a"], d["b"], scale=d["scale"], residual=d["res_y"][p])
    assert torch.equal(y[p], y2) and torch.equal(t[p], t2)


def test_repeatable(tbn):
    # the same bits from every call, ragged and whole (a wait too few would show here)
    for rank, c, k in ((100, 200, 136), (128, 512, 768), (65, 136, 200), (5, 72, 40)):
        for rows in (5, 90):
            d = gpu(make(rows, c, k, rank, 3))
            outs = []
            for _ in range(4):
                y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])
                outs.append((y, t) + tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"]))
            assert all(torch.equal(p, q) for o in outs[1:] for p, q in zip(outs[0], o))


def test_wide(tbn):
    # many splits of the long sums, single tokens
    for rows in (1, 20):
        run(tbn, make(rows, 8192, 4104, 16, 7, index=torch.arange(rows) % 8 - 1))


def test_rows_and_adapters_do_not_mix(tbn):
    # NaN in one adapter or row reaches neither other rows nor other adapters' gradients
    index = torch.tensor([0, 1, 2, 1, 0, -1, 2, 2, 1, 0] * 7)
    for rows in (10, 70):
        s = make(rows, 72, 56, 8, 3, index=index[:rows])
        clean = run(tbn, s)
        s["a"][1, 2, 5] = s["b"][1, 3, 4] = float("nan")
        s["x"][6, 7], s["dy"][0, 0], s["dy"][5] = float("inf"), float("nan"), float("nan")  # rows of adapters 2, 0, none
        d = gpu(s)
        y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])
        keep = [i for i in range(rows) if index[i] != 1 and i != 6]
        assert torch.equal(y[keep], clean[0][keep]) and torch.equal(t[keep], clean[1][keep])
        dx, da, db = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], clean[1], scale=d["scale"], residual=d["res_x"])
        keep = [i for i in range(rows) if index[i] != 1 and i != 0]
        assert torch.equal(dx[keep], clean[2][keep])
        # adapter 1's own gradients need dt = dy B (NaN in b) for da, not for db; adapter 2's da has row 6's infinity
        assert torch.equal(db[1:], clean[4][1:])
        assert torch.isfinite(da[2][:, [c for c in range(72) if c != 7]]).all() and not torch.isfinite(da[2][:, 7]).any()


def test_gradient_by_differences(tbn):
    # the sum of y w is bilinear in x, a and b: central differences are exact but for rounding, 2^-15 |value| / h
    s = make(6, 24, 20, 4, 2, F, F, F, index=torch.tensor([0, 1, 1, -1, 0, 1]))
    d = gpu(s)
    w = d["dy"]
    _, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"])
    grads = tbn.adapter_bwd(d["x"], w, d["index"], d["a"], d["b"], t, scale=d["scale"], out_dtype=F)

    def value(x, a, b):
        y, _ = tbn.adapter_fwd(x, d["index"], a, b, scale=d["scale"], out_dtype=F)
        return float((y.double() * w.double()).sum())

    for k, (name, g) in enumerate(zip(("x", "a", "b"), grads)):
        for i in range(0, d[name].numel(), 7):
            args = [d[n].clone() for n in ("x", "a", "b")]
            args[k].view(-1)[i] += 0.5
            up = value(*args)
            args[k].view(-1)[i] -= 1.0
            assert abs(up - value(*args) - float(g.reshape(-1)[i])) < 2e-2


def test_beside_the_projection(tbn):
    # act(alpha (x W~) + bias + residual + adapters): the adapters' y is the projection's residual
    s = make(48, 128, 192, 8, 4)
    d = gpu(s)
    codes, alpha, _ = tbn.quantize(torch.randn(192, 128, generator=torch.Generator().manual_seed(1)).cuda())
    bias = torch.linspace(-1, 1, 192).cuda()
    x = d["x"].view(48, 1, 1, 128)
    y, _ = tbn.adapter_fwd(x, d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"].float(), out_dtype=F)
    assert y.shape == (48, 1, 1, 192)
    desc = tbn.ConvDesc(48, 1, 1, 128, 192, 1, 1)
    base = tbn.conv2d_fwd(desc, x, codes, alpha, out_dtype=F, bias=bias)
    out = tbn.conv2d_fwd(desc, x, codes, alpha, out_dtype=F, bias=bias, residual=y, relu=True)
    want = (base.double() + y.double()).clamp(min=0)
    assert (out.double() - want).abs().max() <= 4 * U * (base.abs().max() + y.abs().max())


def test_in_place_given_outputs_and_no_dx(tbn):
    s = make(33, 64, 48, 8, 3)
    d = gpu(s)
    y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], residual=d["res_y"])
    same = d["res_y"].clone()
    z, none = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], residual=same, y=same, want_t=False)
    assert z.data_ptr() == same.data_ptr() and torch.equal(z, y) and none is None
    dx, da, db = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t)
    ga, gb = torch.full_like(da, 3.0), torch.full_like(db, 3.0)
    no, ga2, gb2 = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, need_dx=False, da=ga, db=gb)
    assert no is None and ga2.data_ptr() == ga.data_ptr() and torch.equal(ga, da) and torch.equal(gb, db)


def test_other_stream_and_captured(tbn):
    s = make(64, 256, 192, 8, 5)
    d = gpu(s)

    def step():
        y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])
        return (y, t) + tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"], residual=d["res_x"])

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2, 3):  # other rows, other adapters
        new = make(64, 256, 192, 8, 5, seed=seed)
        for f in ("x", "index", "dy"):
            d[f].copy_(new[f])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))


@pytest.mark.parametrize("rows,bank", [(300, 1), (1500, 12), (40, 12)])
def test_in_place_and_captured_at_every_length(tbn, rows, bank):
    # residuals overwritten by the results, by few rows, by rows as they lie and by sorted ones; replays with other adapters
    s = make(rows, 256, 192, 8, bank)
    d = gpu(s)

    def step(y, dx):
        _, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=y, y=y)
        dx, da, db = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"], residual=dx)
        return y, t, dx, da, db

    apart = lambda: tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"])  # noqa: E731
    assert torch.equal(apart()[0], step(d["res_y"].clone(), d["res_x"])[0])
    y = d["res_y"].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step(y, d["res_x"])
    for seed in (1, 2, 3):
        new = make(rows, 256, 192, 8, bank, seed=seed)
        d["x"].copy_(new["x"])
        d["index"].copy_(torch.flip(new["index"], [0]) if seed == 2 else new["index"])
        y.copy_(d["res_y"])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step(d["res_y"].clone(), d["res_x"])))
