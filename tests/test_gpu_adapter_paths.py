"""Low-rank adapters on the paths that a batch's length, its bank and its widths choose, against the formulas in 64 bits: rows taken in
the order of their adapters (more than 8 adapters, more than 1024 rows) at every rank and type and with several splits, the
widest tiles of the expansion, few rows at high ranks for equal bits, and contractions so short that every part of a 32-bit
factor shows.

test_gpu_adapter.py has the tolerances of the long sums; its batches over banks of 1 to 3 are taken as they lie.
"""
import pytest
import torch

import test_gpu_adapter as base
from test_gpu_adapter import BF, F, U

pytestmark = pytest.mark.gpu


def scattered(rows, bank, seed=0):
    """Each row an adapter by chance, some none, one adapter (bank // 2) without rows."""
    index = torch.randint(-2, bank + 2, (rows,), generator=torch.Generator().manual_seed(seed))
    index[index == bank // 2] = -1
    return index


def run_sorted(tbn, rows, c, k, rank, bank, wt=BF, xt=BF, ot=BF):
    s = base.make(rows, c, k, rank, bank, wt, xt, ot, index=scattered(rows, bank, rank))
    _, _, _, da, db = base.run(tbn, s)
    assert not da[bank // 2].any() and not db[bank // 2].any()


@pytest.mark.parametrize("rank", [1, 7, 16, 17, 32, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("wt", [BF, F])
def test_sorted_rows_of_every_rank(tbn, rank, wt):
    run_sorted(tbn, 1030, 136, 72, rank, 12, wt)


@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("xt", [BF, F])
@pytest.mark.parametrize("ot", [BF, F])
@pytest.mark.parametrize("rank", [16, 32, 40])
def test_sorted_rows_of_every_type(tbn, wt, xt, ot, rank):
    run_sorted(tbn, 1100, 168, 90, rank, 17, wt, xt, ot)


@pytest.mark.parametrize("rank,wt,xt", [(16, BF, BF), (32, F, BF), (40, BF, F), (64, F, F), (72, BF, BF), (128, F, BF)])
def test_sorted_rows_with_splits(tbn, rank, wt, xt):
    # both long sums split over blocks (512 values a block at least), the widths ragged and whole
    run_sorted(tbn, 1030, 2056, 2560, rank, 12, wt, xt)


@pytest.mark.parametrize("rank", [8, 40])
@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("bank,c,k", [(1, 7304, 7424), (12, 7424, 7304)])
def test_widest_tiles(tbn, rank, wt, bank, c, k):
    # 9 tiles of 128 rows times 115 or 116 groups of 64 columns, from 1024 on: 256 columns a block up to rank 32, 128 up to 64
    index = scattered(1030, bank, rank) if bank > 1 else None  # runs of rows with and without the one adapter
    base.run(tbn, base.make(1030, c, k, rank, bank, wt, index=index))


@pytest.mark.parametrize("rank", [65, 96, 97, 100, 127, 128])
@pytest.mark.parametrize("wt", [BF, F])
@pytest.mark.parametrize("xt,ot", [(BF, BF), (F, F)])
def test_few_rows_of_high_ranks_repeat(tbn, rank, wt, xt, ot):
    # right, and the same bits from every call, with other work on the card between them
    for rows, c, k in ((5, 200, 136), (40, 513, 72), (90, 136, 1001), (48, 512, 768)):
        s = base.make(rows, c, k, rank, 5, wt, xt, ot, index=scattered(rows, 5, rows))
        d = base.gpu(s)
        first = base.run(tbn, s)
        for n in range(6):
            torch.randn(1000 * (n + 1), device="cuda").sort()
            y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], residual=d["res_y"], out_dtype=ot)
            out = (y, t) + tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t, scale=d["scale"], residual=d["res_x"],
                                           out_dtype=ot)
            assert all(torch.equal(p, q) for p, q in zip(first, out)), (rows, c, k, n)


# Short contractions.  A 32-bit factor is the sum of three bf16 numbers, each at most 2^-8 of the one before, exactly (24 bits are
# 8 + 8 + 8); the product of two leaves out mid lo, lo mid and lo lo: 2 * 2^-24 + 2^-32 of it, 2.1 U.  The parts' products are
# added smallest first, so that only the last MFMA's additions count in full, n + 1 of them (the parts before have 2^-8 of
# its size, six MFMAs of them: 6 (n + 1) 2^-8 of a rounding), each off by a whole step at most, 2 U, of the sum of magnitudes.  With the scale's
# rounding and the sums over waves and tiles (n / 16 and 4 at most): below (2 (min(n, 32) + 1) + n / 16 + 12) U.
# Without its third part a factor is off by up to 2^-16, 256 U, which for n up to 8 this sees in some of many sums (asserted below).
def off(n):
    return (2 * (min(n, 32) + 1) + n / 16 + 12) * U


def two_parts(v):
    hi = v.bfloat16().float()
    return hi.double() + (v - hi).bfloat16().double()


@pytest.mark.parametrize("rows,bank", [(48, 6), (130, 1), (1100, 12)])  # few rows, as they lie, in the adapters' order
@pytest.mark.parametrize("n", [1, 3, 8])
@pytest.mark.parametrize("wt,xt", [(F, F), (F, BF), (BF, F), (BF, BF)])
def test_every_part_of_32_bit_factors(tbn, rows, bank, n, wt, xt):
    s = base.make(rows, n, n, n, bank, wt, xt, F, index=torch.arange(rows) % bank)
    d = base.gpu(s)
    i = s["index"].long()
    x, dy, a, b = s["x"].double(), s["dy"].double(), s["a"].double()[i], s["b"].double()[i]
    sc = s["scale"].double()[i][:, None]

    def times(m, v):  # row by row
        return (m @ v[:, :, None])[:, :, 0]

    y, t = tbn.adapter_fwd(d["x"], d["index"], d["a"], d["b"], scale=d["scale"], out_dtype=F)
    want, tol = times(a, x), off(n) * times(a.abs(), x.abs())
    base.check(t, want, tol, "t")
    if F in (wt, xt):
        short = times(two_parts(s["a"].float())[i], two_parts(s["x"].float()))
        assert ((short - want).abs() > tol).any()
    t = t.cpu()  # y from the t that the call gives
    want, tol = sc * times(b, t.double()), sc * off(n) * times(b.abs(), t.double().abs())
    base.check(y, want, tol, "y")
    if n > 1 or F in (wt, xt):  # (t is one product of two bf16 numbers otherwise: 16 bits)
        assert ((sc * times(b, two_parts(t)) - want).abs() > tol).any()

    dx, da, db = tbn.adapter_bwd(d["x"], d["dy"], d["index"], d["a"], d["b"], t.cuda(), scale=d["scale"], out_dtype=F)
    bt, at = b.transpose(1, 2), a.transpose(1, 2)
    dt, e_dt = sc * times(bt, dy), sc * off(n) * times(bt.abs(), dy.abs())
    base.check(dx, times(at, dt), times(at.abs(), e_dt + off(n) * dt.abs()), "dx")
    own = torch.nn.functional.one_hot(i, bank).double()
    m = int(own.sum(0).max())  # rows of an adapter
    outer = lambda u, v: torch.einsum("nb,nr,nc->brc", own, u, v)  # noqa: E731
    base.check(da, outer(dt, x), outer(e_dt + off(m) * dt.abs(), x.abs()), "da")
    ts = sc * t.double()
    base.check(db, outer(dy, ts), outer(dy.abs(), off(m) * ts.abs()), "db")


@pytest.mark.parametrize("rows", [1, 50, 1500])  # few rows, and rows in the adapters' order
def test_largest_bank(tbn, rows):
    # 65535 adapters of rank 2, 24 -> 40, the first and the last among those in use, a row beyond the bank's end; the gradients of
    # all others are zero
    bank, rank, c, k = 65535, 2, 24, 40
    g = torch.Generator().manual_seed(rows)
    index = torch.randint(0, bank, (rows,), generator=g)
    index[:5] = torch.tensor([bank - 1, 0, bank, bank - 1, bank - 2])[:rows]
    x, dy = torch.randn(rows, c, generator=g).to(BF), torch.randn(rows, k, generator=g).to(BF)
    a, b = torch.randn(bank, rank, c, generator=g).to(BF), torch.randn(bank, k, rank, generator=g).to(BF)
    scale = torch.rand(bank, generator=g) + 0.5
    d = [v.cuda() for v in (x, dy, index.int(), a, b, scale)]
    y, t = tbn.adapter_fwd(d[0], d[2], d[3], d[4], scale=d[5], out_dtype=F)
    dx, da, db = tbn.adapter_bwd(d[0], d[1], d[2], d[3], d[4], t, scale=d[5], out_dtype=F)
    has = (index < bank).double()[:, None]
    i = index.clamp(max=bank - 1)
    x, dy, a, b, sc = x.double(), dy.double(), a[i].double(), b[i].double(), scale[i].double()[:, None] * has

    def times(m, v):
        return (m @ v[:, :, None])[:, :, 0]

    want, tol = times(a, x) * has, off(c) * times(a.abs(), x.abs())
    base.check(t, want, tol, "t")
    t = t.cpu().double()
    base.check(y, sc * times(b, t), sc * off(rank) * times(b.abs(), t.abs()), "y")
    bt, at = b.transpose(1, 2), a.transpose(1, 2)
    dt, e_dt = sc * times(bt, dy), sc * off(k) * times(bt.abs(), dy.abs())
    base.check(dx, times(at, dt), times(at.abs(), e_dt + off(rank) * dt.abs()), "dx")
    m = int(torch.bincount(i).max())

    def bank_sum(u, v):
        return torch.zeros(bank, u.shape[1], v.shape[1], dtype=torch.float64).index_add_(0, i, u[:, :, None] * v[:, None, :])

    base.check(da, bank_sum(dt, x), bank_sum(e_dt + off(m) * dt.abs(), x.abs()), "da")
    base.check(db, bank_sum(dy, sc * t), bank_sum(dy.abs(), off(m) * sc * t.abs()), "db")
