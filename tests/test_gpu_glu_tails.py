"""The gated block's activations where they are small: every value relative to itself, over every gate that bf16 holds and over fp32 gates.

Tolerances.  silu: e^-|g| is the hardware's 2^x (a step, 2^-23) of a product whose rest multiplies it (2^-24); 1 + e^-|g| is rounded (2^-24), its
reciprocal the hardware's (2^-23), and two products follow, a third by u: at most 1.5 + 0.5 + 1 + 1.5 = 4.5 steps of 2^-23.  gelu is
held to 18.5: the 16 that an fp32 erfc is commonly specified with, its argument's rest and three products.
What lies below 2^-119 may come as 0: an exponential below 2^-126 times a gate.  The slopes are written in bf16 (2^-8 of the value), before
which each of their terms is off by at most 2^-16 of itself (its exponential's argument, up to 88, is rounded to 2^-24).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
STEP, FLUSHED = 2.0 ** -23, 2.0 ** -119
OFF = {"silu": 4.5 * STEP, "gelu": 18.5 * STEP}


def act64(name, g):
    """(act, the two terms of its slope), relative to themselves also in the tails."""
    if name == "silu":
        s = torch.exp(-g.abs()) / (1 + torch.exp(-g.abs()))  # of -|g|
        s, other = torch.where(g < 0, s, 1 - s), torch.where(g < 0, 1 - s, s)
        return g * s, s, g * s * other
    phi = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * phi, phi, g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_every_gate(tbn, act):
    g = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF).cuda()
    g = torch.where(torch.isfinite(g), g, torch.zeros_like(g)).view(64, -1)
    gu = torch.cat([g, torch.ones_like(g)], 1)
    dgu, h = tbn.glu_bwd(torch.ones_like(g), gu=gu, act=act, want_h=True, out_dtype=F)
    a, first, second = act64(act, g.double())
    off = (h.double() - a).abs()
    assert bool((off <= OFF[act] * a.abs() + FLUSHED).all()), (off / a.abs())[off > FLUSHED].max().item()
    dg, du = dgu.double().chunk(2, 1)
    assert bool(((du - a).abs() <= (2.0 ** -8 + 2.0 ** -16) * a.abs() + FLUSHED).all())
    slope = first + second
    assert bool(((dg - slope).abs() <= 2.0 ** -8 * slope.abs() + 1.01 * 2.0 ** -16 * (first + second.abs()) + FLUSHED).all())


def test_gates_that_are_not_finite(tbn):
    gate = torch.tensor([[math.inf, -math.inf, math.nan]], device="cuda").to(BF)
    gu = torch.cat([gate, torch.ones_like(gate)], 1)
    for act in ("silu", "gelu", "relu"):
        h = tbn.glu_bwd(torch.ones_like(gate), gu=gu, act=act, want_h=True, out_dtype=F)[1][0]
        assert h[0] == math.inf and torch.isnan(h[2])
        assert h[1] == 0 if act == "relu" else torch.isnan(h[1])  # -inf times 0


# rows, c, f: x in registers, read with the codes, tiles
@pytest.mark.parametrize("rows,c,f", [(16, 8, 40), (9, 8208, 24), (2000, 8, 24)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_fp32_gates_of_the_forward_pass(tbn, rows, c, f, act):
    """One feature that is not zero, codes of 1: g is a product of two numbers, rounded once, u the feature itself."""
    codes = tbn.quantize(torch.full((2 * f, c), 0.5, device="cuda"))[0]
    gen = torch.Generator().manual_seed(1)
    alpha = torch.cat([0.5 + torch.rand(f, generator=gen), torch.ones(f)]).cuda()
    x = torch.zeros(rows, c, dtype=BF)
    x[:, c // 3] = torch.linspace(-57.0 if act == "silu" else -8.5, 4.0, rows)
    x = x.cuda()
    h = tbn.glu_fwd(x, codes, alpha, act=act, out_dtype=F)[0]
    g = (x[:, c // 3:c // 3 + 1].float() * alpha[:f]).double()
    want = act64(act, g)[0] * x[:, c // 3:c // 3 + 1].double()
    off = (h.double() - want).abs()
    assert bool((off <= OFF[act] * want.abs() + 57 * FLUSHED).all()), (off / want.abs())[off > 57 * FLUSHED].max().item()
