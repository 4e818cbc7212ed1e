"""Muon's step against its formulas in 64 bits: shapes on every tile and on divided tiles, tall and wide, many matrices at once.

Tolerance of the orthogonalised update O, |O - O64| in the Frobenius norm.  A factor held in 22 bits is off by 2^-22 of each value, so is a
product without its lo lo term, and a sum in fp32 by less: a product of m x m by X is off by at most 2^-21 sqrt(m) |P| |X| (spectral
norm of P, Frobenius norms else).  Such an error in X grows by at most a = 3.4445 a step.  One in the Gram matrix, 2^-21 of |X|^2 <= 1.5, goes into
P times |p'| <= 4.8, after a further step on the same product times 4.8 a^2 = 57.  With |X0| = 1 and `k` steps each of some ten
roundings adds at most 3 a^k 2^-21 sqrt(m) (57 a^(k - 2) < 5 a^k): 64 2^-21 sqrt(m) a^k in all.  That bounds the worst spectrum; a wrong
coefficient, scale or tile is off by the size of O itself.  The usual spectra are held to 1e-4 of |O| beside it.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
A, B, C = 3.4445, -4.7750, 2.0315


def orthogonal64(u, steps, eps=1e-7):
    x = u / (u.norm() + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(steps):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.t() if tall else x


def case(rows, cols, seed=0, dtype=F, kind="noise"):
    g = torch.Generator().manual_seed(seed * 1000003 + rows * 1009 + cols)
    few = max(1, min(rows, cols) // 16)
    low = torch.randn(rows, few, generator=g) @ torch.randn(few, cols, generator=g)
    grad = (0.3 * low if kind == "low" else 0) + torch.randn(rows, cols, generator=g)
    w, m = torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g) * 2
    return w.cuda(), m.cuda(), grad.to(dtype).cuda()


def check(w, m, w0, m0, g, lr, momentum=0.95, nesterov=True, wd=0.0, scale=None, steps=5, eps=1e-7):
    g64, m64 = g.double().view(g.shape[0], -1), m0.double().view(g.shape[0], -1)
    m64 = momentum * m64 + g64
    u = g64 + momentum * m64 if nesterov else m64
    o = orthogonal64(u, steps, eps)
    rows, cols = o.shape
    scale = max(1.0, rows / cols) ** 0.5 if scale is None else scale
    m, w, w0 = (t.view(rows, -1) for t in (m, w, w0))
    # momentum: two roundings, and the factor's to fp32
    assert ((m.double() - m64).abs() <= 3 * 2.0 ** -24 * (momentum * m0.double().view(rows, -1).abs() + g64.abs())).all()
    want = w0.double() * (1 - lr * wd) - lr * scale * o
    off = (w.double() - want).norm().item()
    small = min(rows, cols)
    rounding = 4 * 2.0 ** -24 * (w0.double().norm().item() + lr * scale * o.norm().item())
    worst = 64 * 2.0 ** -21 * small ** 0.5 * A ** steps
    assert torch.isfinite(w).all()
    assert off <= lr * scale * worst + rounding, (off, worst)
    assert off <= lr * scale * 1e-4 * o.norm().item() + rounding, (off / (lr * scale * o.norm().item()))


SHAPES = [(1, 1), (1, 9), (9, 1), (2, 3), (31, 32), (33, 31), (32, 25), (10, 512), (512, 10), (64, 64), (65, 63), (64, 147), (129, 77), (77, 300),
          (200, 1000), (1000, 130), (500, 500), (512, 1153), (1031, 517)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F, BF])
def test_step(tbn, rows, cols, dtype):
    w, m, g = case(rows, cols, dtype=dtype)
    w0, m0 = w.clone(), m.clone()
    out = tbn.muon_step([w], [m], [g], lr=0.5, weight_decay=0.1)
    assert out[0][0] is w and out[1][0] is m
    check(w, m, w0, m0, g, 0.5, wd=0.1)


@pytest.mark.parametrize("rows,cols", [(1500, 2600), (2304, 1100), (300, 20000), (4096, 2048), (3000, 4100)])
def test_large(tbn, rows, cols):
    w, m, g = case(rows, cols, kind="low")
    w0, m0 = w.clone(), m.clone()
    tbn.muon_step([w], [m], [g], lr=0.5)
    check(w, m, w0, m0, g, 0.5)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
@pytest.mark.parametrize("rows,cols", [(40, 100), (100, 40)])
def test_steps(tbn, steps, rows, cols):
    w, m, g = case(rows, cols)
    w0, m0 = w.clone(), m.clone()
    tbn.muon_step([w], [m], [g], lr=0.5, steps=steps)
    check(w, m, w0, m0, g, 0.5, steps=steps)


def test_the_most_steps(tbn):
    # many steps settle: singular values between 0.7 and 1.2 (the polynomial's range around 1)
    w, m, g = case(48, 64)
    w.zero_()
    tbn.muon_step([w], [m], [g], lr=1.0, steps=32)
    s = torch.linalg.svdvals(w.double())
    assert s.min() > 0.65 and s.max() < 1.25


def test_hyperparameters(tbn):
    w, m, g = case(70, 90)
    for kw in ({"nesterov": False}, {"momentum": 0.0}, {"momentum": 0.5, "nesterov": False}, {"scale": 0.3}, {"wd": 0.7}, {"eps": 1.0}):
        w1, m1 = w.clone(), m.clone()
        call = {("weight_decay" if k == "wd" else k): ([v] if k == "scale" else v) for k, v in kw.items()}
        tbn.muon_step([w1], [m1], [g], lr=0.25, **call)
        check(w1, m1, w, m, g, 0.25, **kw)
    w1, m1, w2, m2 = w.clone(), m.clone(), w.clone(), m.clone()
    tbn.muon_step([w1], [m1], [g], lr=torch.full((1,), 0.25, device="cuda"))
    tbn.muon_step([w2], [m2], [g], lr=0.25)
    assert torch.equal(w1, w2) and torch.equal(m1, m2)


@pytest.mark.parametrize("kind", ["rank one", "decay", "tiny", "huge"])
def test_spectra(tbn, kind):
    """Where small singular values carry what rounding left, the worst-case bound alone holds; the strong directions are as good as ever."""
    g = torch.Generator().manual_seed(9)
    u, _ = torch.linalg.qr(torch.randn(96, 96, generator=g, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(200, 96, generator=g, dtype=torch.float64))
    s = {"rank one": torch.tensor([1.0] + [0.0] * 95), "decay": torch.logspace(0, -5, 96), "tiny": torch.full((96,), 1e-20),
         "huge": torch.full((96,), 1e20)}[kind].double()
    grad = ((u * s) @ v.t()).float().cuda()
    w, m = torch.zeros(96, 200, device="cuda"), torch.zeros(96, 200, device="cuda")
    tbn.muon_step([w], [m], [grad], lr=1.0, momentum=0.0, nesterov=False, eps=1e-30)
    o = orthogonal64(grad.double(), 5, 1e-30)
    assert (-w.double() - o).norm() <= 64 * 2.0 ** -21 * 96 ** 0.5 * A ** 5
    strong = (u[:, :10].cuda().t() @ (-w.double() - o) @ v[:, :10].cuda()).norm()
    if kind != "rank one":
        assert strong <= 1e-4 * 10 ** 0.5


def test_no_update_moves_nothing_but_the_decay(tbn):
    w = torch.randn(30, 50, device="cuda")
    w0, m, g = w.clone(), torch.zeros(30, 50, device="cuda"), torch.zeros(30, 50, device="cuda")
    tbn.muon_step([w], [m], [g], lr=0.5, weight_decay=0.5)
    assert torch.equal(w, w0 * 0.75) and not m.any()


def test_many_matrices_at_once_are_as_if_alone(tbn):
    """More than share a launch, of all shapes, in buffers of any alignment."""
    g = torch.Generator().manual_seed(2)
    sides = [(int(torch.randint(1, 150, (1,), generator=g)), int(torch.randint(1, 150, (1,), generator=g))) for _ in range(70)] + [(512, 600), (600, 512)]
    n = sum(r * c for r, c in sides) + len(sides)
    flat = [torch.randn(n, generator=g).cuda() for _ in range(3)]
    lists, at = [[], [], []], 0
    for i, (r, c) in enumerate(sides):
        for l, f in zip(lists, flat):
            l.append(f[at:at + r * c].view(r, c))
        at += r * c + i % 2  # odd places among them
    w0, m0 = flat[0].clone(), flat[1].clone()
    before = [[t.clone() for t in l] for l in lists]
    decays, scales = [0.01 * (i % 3) for i in range(len(sides))], [1.0 + i % 4 for i in range(len(sides))]
    tbn.muon_step(*lists, lr=0.5, weight_decay=decays, scale=scales)
    for i in range(len(sides)):
        check(lists[0][i], lists[1][i], before[0][i], before[1][i], lists[2][i], 0.5, wd=decays[i], scale=scales[i])
    # what lies between the matrices is as it was
    mask = torch.ones(n, dtype=torch.bool, device="cuda")
    at = 0
    for i, (r, c) in enumerate(sides):
        mask[at:at + r * c] = False
        at += r * c + i % 2
    assert torch.equal(flat[0][mask], w0[mask]) and torch.equal(flat[1][mask], m0[mask])


def test_filters_of_a_convolution(tbn):
    w, m, g = case(16, 3 * 3 * 8)
    shaped = [t.clone().view(16, 3, 3, 8) for t in (w, m, g)]
    tbn.muon_step([w], [m], [g])
    tbn.muon_step([shaped[0]], [shaped[1]], [shaped[2]])
    assert torch.equal(shaped[0].view(16, -1), w) and torch.equal(shaped[1].view(16, -1), m)


def test_what_is_not_finite_stays_in_its_matrix(tbn):
    cases = [case(60, 80, seed=s) for s in range(3)]
    clean = [[t.clone() for t in c] for c in cases]
    tbn.muon_step(*[[c[k] for c in clean] for k in range(3)])
    for v in (float("nan"), float("inf")):
        got = [[t.clone() for t in c] for c in cases]
        got[1][2][3, 5] = v
        tbn.muon_step(*[[c[k] for c in got] for k in range(3)])
        for i in (0, 2):
            assert torch.equal(got[i][0], clean[i][0]) and torch.equal(got[i][1], clean[i][1])
        assert torch.isnan(got[1][0]).all()
        assert not torch.isfinite(got[1][1][3, 5]) and torch.isfinite(got[1][1]).sum() == 60 * 80 - 1


@pytest.mark.parametrize("rows,cols", [(100, 200), (512, 3136), (700, 4000)])
def test_same_bits_from_call_to_call(tbn, rows, cols):
    w, m, g = case(rows, cols)
    first = None
    for _ in range(6):
        w1, m1 = w.clone(), m.clone()
        tbn.muon_step([w1], [m1], [g])
        assert first is None or (torch.equal(first[0], w1) and torch.equal(first[1], m1))
        first = (w1, m1)


def test_workspace_beyond_4_gib(tbn):
    """Arrays that begin, and end, past 32 bits of the workspace."""
    rows, cols = 256, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(4)
    grad = torch.empty(rows, cols, device="cuda").normal_(generator=g)
    w, m = torch.zeros(rows, cols, device="cuda"), torch.zeros(rows, cols, device="cuda")
    assert tbn.muon_workspace_size([w]) > 1 << 32
    tbn.muon_step([w], [m], [grad], lr=1.0)
    u = grad.double() * 1.95
    u /= u.norm() + 1e-7
    for _ in range(5):
        gram = u @ u.t()
        u = (A * torch.eye(rows, device="cuda", dtype=torch.float64) + B * gram + C * (gram @ gram)) @ u
    assert (w.double() + u).norm() <= 1e-4 * u.norm()
