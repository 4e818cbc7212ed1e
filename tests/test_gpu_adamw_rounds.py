"""AdamW whose blocks take several rounds of 1024 elements, against the formulas in 64 bits (the lists of test_gpu_adamw.py have up to
70001 elements: a round a block), and what an infinite gradient does.
"""
import pytest
import torch

import test_gpu_adamw as adamw

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32

# rounds of 1024: 512 to 1023 of them are two a block, from 1024 on four.  Tensors that end in each round of a block, at its
# end, in a scale's 256 elements, and such that are shorter than a block
ROUNDS = [[600001, 5], [1024 * 512], [300 * 2048, 2047, 1025], [1100003, 3, 70001, 4097], [300 * 4096], [1024 * 1021 + 1, 2049, 3073, 255],
          [500000] * 3 + [1] * 70]


@pytest.mark.parametrize("gt", [F, BF])
@pytest.mark.parametrize("sizes", ROUNDS, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_adamw_32_bits_in_rounds(tbn, sizes, gt):
    adamw.test_32_bits(tbn, sizes, gt)


@pytest.mark.parametrize("gt", [F, BF])
@pytest.mark.parametrize("sizes", ROUNDS, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_adamw_8_bits_in_rounds(tbn, sizes, gt):
    adamw.test_8_bits(tbn, sizes, gt)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_infinite_gradient(tbn, bits):
    # m and v are infinite, and the step, their quotient, is NaN; the neighbours move as they do without it
    for n in (600, 1300000):
        g = torch.full((n,), 0.01)
        g[300] = float("inf")
        w = [torch.ones(n, device="cuda")]
        m, v, ms, vs = tbn.adamw_state(w[0], bits=bits)
        kw = {} if bits == 32 else {"m_scale": [ms], "v_scale": [vs]}
        tbn.adamw_step(w, [m], [v], [g.cuda()], 1, weight_decay=0.0, **kw)
        assert torch.isnan(w[0][300])
        assert torch.isinf(m[300]) and torch.isinf(v[300]) if bits == 32 else torch.isnan(m.float()[300]) and torch.isnan(v.float()[300])
        rest = torch.cat([w[0][:300], w[0][301:]])
        # lr m / (sqrt v + eps) = 1e-3 (1 - eps / 0.01): a dozen roundings of the step, one of w
        assert (rest.double() - (1 - 1e-3 * (1 - 1e-6))).abs().max() < 20 * U * 1e-3 + U
