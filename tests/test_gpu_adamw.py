"""AdamW over many tensors against the formula in 64 bits; 8-bit states also against their rounding rule, code by code.

Tolerances, from u = 2^-24: m and v are two fp32 roundings of what is added, the step's quotient a dozen (division, roots,
factors formed in fp32), w two of its own.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HYPER = {"lr": 3e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8}
BLOCK = 256


def tensors(sizes, seed, gt=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return ([torch.randn(n, generator=g) for n in sizes], [(torch.randn(n, generator=g) * 0.02).to(gt) for n in sizes])


def formula(w, m, v, g, step, wd, lr, beta1, beta2, eps):
    w, m, v, g = (t.double() for t in (w, m, v, g))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    move = lr * (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps)
    return w - lr * wd * w - move, m, v, move


def check(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol
    assert not torch.isnan(off).any() and off.max() <= 0, "%s: %g over the tolerance" % (what, off.max())


def check_w(w, w0, m0, v0, g, step, wd, hyper=HYPER):
    want, m, v, move = formula(w0, m0, v0, g, step, wd, **hyper)
    # the move's relative error: that of m (its terms may cancel) and a dozen roundings
    m_off = 3 * U * (m0.double().abs() + g.double().abs()) * hyper["lr"] / (1 - hyper["beta1"] ** step)
    check(w, want, 4 * U * w0.double().abs() + 2 * U * want.abs() + 20 * U * move.abs() +
          m_off / ((v / (1 - hyper["beta2"] ** step)).sqrt() + hyper["eps"]) + 1e-45, "w")
    return m, v


@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[1], [2, 3, 5], [255, 256, 257, 4095, 4096, 4097], [70001], [17] * 130])
def test_32_bits(tbn, sizes, gt):
    w, _ = tensors(sizes, 1)
    w0 = [t.clone() for t in w]
    w = [t.cuda() for t in w]
    m, v = zip(*[tbn.adamw_state(t)[:2] for t in w])
    m, v = list(m), list(v)
    decays = [0.1 if i % 2 else 0.0 for i in range(len(w))]
    for step in (1, 2, 3):
        g = tensors(sizes, 10 + step, gt)[1]
        m0, v0 = [t.cpu() for t in m], [t.cpu() for t in v]
        out = tbn.adamw_step(w, m, v, [t.cuda() for t in g], step, weight_decay=decays, **HYPER)
        assert out[0] is w
        for i in range(len(w)):
            mm, vv = check_w(w[i], w0[i], m0[i], v0[i], g[i], step, decays[i])
            check(m[i], mm, 3 * U * (m0[i].double().abs() + g[i].double().abs()) + 1e-45, "m")
            check(v[i], vv, 5 * U * vv + 1e-45, "v")
        w0 = [t.cpu() for t in w]


def mix(h):
    h = np.asarray(h, dtype=np.uint64) & 0xFFFFFFFF
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    return h ^ (h >> np.uint64(16))


def check_codes(codes, scale, want, off, rnd, what):
    """Codes and scales of `want` (64 bits, `off`: how far its fp32 value may be): the scale is the block's top / 448; a
    code is the value over it, rounded up where the random number (of 20 bits) carries.  Within `off` and the
    roundings of the division (16 steps at most, 4 u each) of the carry, fp32 may decide otherwise."""
    n = want.numel()
    blocks = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=torch.float64)
    blocks[:n] = want
    top = blocks.view(-1, BLOCK).abs().amax(1)
    check(scale, top / 448, (float(off.max()) + 8 * U * top) / 448, what + " scale")
    x = (want / (top / 448).repeat_interleave(BLOCK)[:n]).nan_to_num().numpy()
    a = np.abs(x)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-30))), -6) - 3)
    at = a / step + rnd / 2.0 ** 20
    got = codes.cpu().float().double().numpy()
    slack = (off / (top / 448).repeat_interleave(BLOCK)[:n]).nan_to_num().numpy() / step + 64 * U + 2 * float((off.max() / top).max()) * 16
    assert (np.sign(got) * np.sign(x) >= 0)[a > step * slack].all()
    sure = np.abs(at - np.round(at)) > slack
    # (a value that is rounded up to a power of two begins a range of longer steps there: the same value)
    expected = np.minimum(np.floor(at) * step, 448)
    assert (np.abs(got)[sure] == expected[sure]).all(), what
    assert (np.abs(got - x) <= step * (1 + slack)).all()
    assert sure.mean() > 0.95 or n < 300


@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[1], [3, 255, 256, 257], [4095, 4096, 4097, 6], [66001], [19] * 130])
def test_8_bits(tbn, sizes, gt):
    w, _ = tensors(sizes, 2)
    w0 = [t.clone() for t in w]
    w = [t.cuda() for t in w]
    m, v, ms, vs = (list(l) for l in zip(*[tbn.adamw_state(t, bits=8) for t in w]))
    seed = 12345
    for step in (1, 2, 700):
        g = tensors(sizes, 20 + step, gt)[1]

        def decoded(c, s, i):
            return (c[i].float() * s[i].repeat_interleave(BLOCK)[:sizes[i]]).cpu()

        m0 = [decoded(m, ms, i) for i in range(len(w))]
        r0 = [decoded(v, vs, i) for i in range(len(w))]
        tbn.adamw_step(w, m, v, [t.cuda() for t in g], step, weight_decay=0.05, m_scale=ms, v_scale=vs, seed=seed, **HYPER)
        for i in range(len(w)):
            mm, vv = check_w(w[i], w0[i], m0[i], r0[i].double() ** 2, g[i], step, 0.05)
            key = mix(mix(mix(seed) ^ np.uint64(step)) ^ np.uint64(i))
            h = mix(np.arange(sizes[i], dtype=np.uint64) ^ key)
            m_off = 3 * U * (m0[i].double().abs() + g[i].double().abs())
            check_codes(m[i], ms[i], mm, m_off, (h & np.uint64(0xFFFFF)).astype(np.float64), "m")
            check_codes(v[i], vs[i], vv.sqrt(), 5 * U * vv.sqrt(), (h >> np.uint64(12)).astype(np.float64), "root of v")
        w0 = [t.cpu() for t in w]


def test_rounding_by_chance_is_fair(tbn):
    # the mean rounding error over n values is below 5 standard deviations: each is at most half a step (variance 1/4)
    n = 1 << 16
    w = [torch.zeros(n, device="cuda")]
    m, v, ms, vs = ([t] for t in tbn.adamw_state(w[0], bits=8))
    g = [(torch.randn(n, generator=torch.Generator().manual_seed(4)) * 0.1).cuda()]
    tbn.adamw_step(w, m, v, g, 1, m_scale=ms, v_scale=vs, seed=99)
    for c, s, want in ((m[0], ms[0], 0.1 * g[0].double()), (v[0], vs[0], math.sqrt(0.001) * g[0].double().abs())):
        x = want / s.double().repeat_interleave(BLOCK)
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=1e-30))).clamp(min=-6) - 3)
        err = (c.float().double() - x) / step
        assert err.abs().max() < 1.001
        assert abs(float(err.mean())) < 5 * 0.5 / math.sqrt(n)
        assert abs(float((err * x.sign()).mean())) < 5 * 0.5 / math.sqrt(n)


def test_8_bit_moments_follow_small_changes(tbn):
    # the second moment decays by 0.1% a step, a sixtieth of a code's step: by chance it arrives on average.  All of a block but
    # its top decay for 200 steps without gradients; the expected root is 0.999^100 of the start, the spread of the mean
    # over 255 * 64 elements below 5 * 0.125 * sqrt(200 * 0.01 * 0.99) / sqrt(255 * 64) of it
    n = 64 * BLOCK
    w = [torch.zeros(n, device="cuda")]
    m, v, ms, vs = ([t] for t in tbn.adamw_state(w[0], bits=8))
    codes = torch.full((n,), 20.0, device="cuda")
    codes[::BLOCK] = 448.0
    v[0].copy_(codes.to(torch.float8_e4m3fn))
    vs[0].fill_(1e-3)
    g = torch.zeros(n, device="cuda")
    for step in range(1, 201):
        g[::BLOCK] = 0.448  # keeps the tops where they are
        tbn.adamw_step(w, m, v, [g], step, lr=0.0, weight_decay=0.0, m_scale=ms, v_scale=vs, seed=5)
    root = (v[0].float() * vs[0].repeat_interleave(BLOCK)).view(-1, BLOCK)[:, 1:].double()
    want = 0.02 * 0.999 ** 100
    assert abs(float(root.mean()) - want) < 5 * 0.125 * 0.02 * math.sqrt(200 * 0.01 * 0.99) / math.sqrt(255 * 64)


def test_non_finite_and_tiny_values(tbn):
    # NaN and infinities stay with their elements; a block of tiny values is kept as zeros
    g = torch.full((600,), 0.01)
    g[5], g[300], g[512:] = float("nan"), float("inf"), 1e-36
    for bits in (32, 8):
        w = [torch.ones(600, device="cuda")]
        m, v, ms, vs = tbn.adamw_state(w[0], bits=bits)
        kw = {} if bits == 32 else {"m_scale": [ms], "v_scale": [vs]}
        tbn.adamw_step(w, [m], [v], [g.cuda()], 1, weight_decay=0.0, **kw)
        bad = [5, 300]
        assert not torch.isfinite(w[0][bad]).any() or bits == 32
        keep = [i for i in range(600) if i not in bad]
        assert torch.isfinite(w[0][keep]).all() and torch.isfinite(m.float()[keep]).all() and torch.isfinite(v.float()[keep]).all()
        assert torch.isnan(w[0][5])
        if bits == 8:
            assert torch.isnan(m.float()[bad]).all() and torch.isnan(v.float()[bad]).all()
            assert float(ms[2]) == 0 and float(vs[2]) == 0 and not m.float()[512:].any()
            assert torch.isfinite(ms).all() and torch.isfinite(vs).all()


def test_views_at_any_alignment(tbn):
    # tensors that begin anywhere in flat buffers; what lies between them stays as it was
    sizes, pad = [1000, 1, 333, 4099], 3
    n = sum(sizes) + pad * (len(sizes) + 1)
    starts = [pad + sum(sizes[:i]) + pad * i for i in range(len(sizes))]
    for bits in (32, 8):
        for gt in (torch.float32, torch.bfloat16):
            w, g = tensors([n], 3)
            flat = [t.cuda() for t in (w[0], g[0].to(gt))]
            cut = lambda t: [t[s:s + k] for s, k in zip(starts, sizes)]  # noqa: E731
            st = [torch.zeros(n, device="cuda") if bits == 32 else torch.zeros(n, dtype=torch.uint8, device="cuda")
                  .view(torch.float8_e4m3fn) for _ in range(2)]
            own = [t.clone() for t in cut(flat[0])]
            state = [tbn.adamw_state(t, bits=bits) for t in own]
            kw, kw2 = ({}, {}) if bits == 32 else (
                {"m_scale": [torch.zeros_like(s[2]) for s in state], "v_scale": [torch.zeros_like(s[3]) for s in state]},
                {"m_scale": [s[2] for s in state], "v_scale": [s[3] for s in state]})
            before = flat[0].clone()
            tbn.adamw_step(cut(flat[0]), cut(st[0]), cut(st[1]), cut(flat[1]), 4, **kw)
            tbn.adamw_step(own, [s[0] for s in state], [s[1] for s in state], [t.clone() for t in cut(flat[1])], 4, **kw2)
            for p, q in zip(cut(flat[0]), own):
                assert torch.equal(p, q)
            for k in range(2):
                for p, q in zip(cut(st[k]), state):
                    assert torch.equal(p.view(torch.uint8) if bits == 8 else p, q[k].view(torch.uint8) if bits == 8 else q[k])
            mask = torch.ones(n, dtype=torch.bool)
            for s, k in zip(starts, sizes):
                mask[s:s + k] = False
            assert torch.equal(flat[0].cpu()[mask], before.cpu()[mask])


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_rate_in_device_memory_and_captured(tbn, bits):
    sizes = [300, 5000, 7]
    w, g = tensors(sizes, 6)

    def fresh():
        p = [t.cuda() for t in w]
        s = [tbn.adamw_state(t, bits=bits) for t in p]
        return p, [x[0] for x in s], [x[1] for x in s], {} if bits == 32 else {"m_scale": [x[2] for x in s], "v_scale": [x[3] for x in s]}

    grads = [t.cuda() for t in g]
    step, lr = torch.ones(1, dtype=torch.int32, device="cuda"), torch.full((1,), 0.01, device="cuda")
    p, m, v, kw = fresh()
    p2, m2, v2, kw2 = fresh()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tbn.adamw_step(p, m, v, grads, step, lr=lr, weight_decay=0.02, **kw)
        step.add_(1)
    for t in range(1, 5):
        rate = 0.01 / t
        lr.fill_(rate)
        for i, x in enumerate(tensors(sizes, 30 + t)[1]):
            grads[i].copy_(x)
        w0, m0 = [x.cpu() for x in p], m
        before = [(x.float() * kw["m_scale"][i].repeat_interleave(BLOCK)[:sizes[i]] if bits == 8 else x.clone()).cpu() for i, x in enumerate(m)]
        root = [(x.float() * kw["v_scale"][i].repeat_interleave(BLOCK)[:sizes[i]] if bits == 8 else x.sqrt()).cpu() for i, x in enumerate(v)]
        second = [(r.double() ** 2 if bits == 8 else x.cpu().double()) for r, x in zip(root, v)]
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == t + 1
        for i in range(3):
            check_w(p[i], w0[i], before[i], second[i], grads[i].cpu(), t, 0.02, dict(HYPER, lr=float(np.float32(rate))))
        # the same step by numbers: factors formed in other ways differ in their last bit
        tbn.adamw_step(p2, m2, v2, grads, t, lr=float(np.float32(rate)), weight_decay=0.02, **kw2)
    for a, b in zip(p, p2):
        assert (a - b).abs().max() < 1e-5


def test_other_stream_and_repeatable(tbn):
    sizes = [100, 9000]
    results = []
    for k in range(2):
        w, g = tensors(sizes, 8)
        w, g = [t.cuda() for t in w], [t.cuda() for t in g]
        s = [tbn.adamw_state(t, bits=8) for t in w]
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream() if k else torch.cuda.current_stream()):
            for step in (1, 2):
                tbn.adamw_step(w, [x[0] for x in s], [x[1] for x in s], g, step, m_scale=[x[2] for x in s], v_scale=[x[3] for x in s])
        torch.cuda.synchronize()
        results.append(w + [x[k].view(torch.uint8) for x in s for k in range(2)] + [x[k] for x in s for k in (2, 3)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_large_step_counts_and_plain_sgd_limits(tbn):
    # far steps: the bias corrections are 1; beta 0: no memory
    w, g = tensors([500], 9)
    for step, hyper in ((2 ** 31 - 1, HYPER), (5, dict(HYPER, beta1=0.0, beta2=0.0))):
        p = [w[0].cuda()]
        m, v, _, _ = tbn.adamw_state(p[0])
        m.fill_(0.01)
        v.fill_(1e-4)
        tbn.adamw_step(p, [m], [v], [g[0].cuda()], step, weight_decay=0.0, **hyper)
        check_w(p[0], w[0], torch.full((500,), 0.01), torch.full((500,), 1e-4), g[0], step, 0.0, hyper)
