"""The operators of a feed-forward block, trained and served, as cases to time and to compare: the gated block over
two-bit filters (forward, and backward from the block's output to the two projections), Muon's step on the real
weights (an update orthogonalised by Newton-Schulz products), and the product in 8-bit integers with a scale for each
token and each channel, for the layers that stay out of two bits.

`run` computes them in their plain form, elementary torch operations in 32 bits, or, where `own` is true, by the
calls of ``paper_1701_00485_amd``.  `exact` says what the definitions give in 64 bits.

Kinds of case (field "kind"):
  glu_fwd    `rows` rows of c features through 2f two-bit filters, f of them gates; "gu": the projections are wanted
             too, for the backward pass
  glu_bwd    the gradient of the 2f projections from that of the f outputs; "from" the projections that the forward
             pass kept ("gu") or the input ("x": they are computed again, and the outputs too, for the next layer's
             gradient)
  muon       the matrices of a network of this repository ("model"), or `matrices` of them whose sides are drawn up to
             `longest` from `pick`; gradients in "f32" or "bf16"
  linear_i8  `rows` rows of c features in bf16, made 8-bit with a scale each, times n channels of 8-bit weights
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, MOMENTUM, EPS, DECAY, STEPS = 0.02, 0.95, 1e-7, 0.01, 5
POLY = (3.4445, -4.7750, 2.0315)  # of the singular values: a s + b s^3 + c s^5, five times


def _resnet18():
    shapes, cin = [(64, 147)], 64
    for cout in (64, 128, 256, 512):
        for block in range(2):
            shapes += [(cout, 9 * cin), (cout, 9 * cout)] + ([(cout, cin)] if block == 0 and cin != cout else [])
            cin = cout
    return shapes + [(1000, 512)]


MODELS = {
    "lenet": [(32, 25), (64, 800), (512, 3136), (10, 512)],
    "resnet18": _resnet18(),
    "up": [(8192, 4096)],  # a projection from 4096 features to 8192
}


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the smallest call: one token of a 512-feature network, latency counts
        {"name": "glu_fwd_1x512", "kind": "glu_fwd", "rows": 1, "c": 512, "f": 1024, "act": "silu", "gu": False},
        # a serving step: one token of each of 16 requests through a large block
        {"name": "glu_fwd_decode16", "kind": "glu_fwd", "rows": 16, "c": 8192, "f": 16384, "act": "silu", "gu": False},
        # a ragged batch over sizes that are no multiples of a tile, in training
        {"name": "glu_fwd_777", "kind": "glu_fwd", "rows": 777, "c": 1000, "f": 1333, "act": "gelu", "gu": True},
        # a large training batch
        {"name": "glu_fwd_8192", "kind": "glu_fwd", "rows": 8192, "c": 4096, "f": 8192, "act": "silu", "gu": True},
        # the gradient of a small batch, from the projections that the forward pass kept
        {"name": "glu_bwd_300", "kind": "glu_bwd", "rows": 300, "c": 512, "f": 2048, "act": "silu", "from": "gu"},
        # ... of a large one that kept its input alone
        {"name": "glu_bwd_8192", "kind": "glu_bwd", "rows": 8192, "c": 4096, "f": 8192, "act": "silu", "from": "x"},
        # the four layers of LeNet: a small model's step
        {"name": "muon_lenet", "kind": "muon", "model": "lenet", "grad": "f32"},
        # the 21 layers of ResNet-18, of 64 to 512 filters
        {"name": "muon_resnet18", "kind": "muon", "model": "resnet18", "grad": "f32"},
        # one large projection, with gradients that a backward pass left in 16 bits
        {"name": "muon_up", "kind": "muon", "model": "up", "grad": "bf16"},
        # a serving step of one token through the 8192 -> 32768 layer
        {"name": "i8_decode1", "kind": "linear_i8", "rows": 1, "c": 8192, "n": 32768, "out": "bf16"},
        # a ragged batch
        {"name": "i8_777", "kind": "linear_i8", "rows": 777, "c": 1000, "n": 1333, "out": "f32"},
        # a long prompt
        {"name": "i8_8192", "kind": "linear_i8", "rows": 8192, "c": 4096, "n": 8192, "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """Mostly multiples of 64, as networks have; one in four as it falls."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.25 else max(64, (c + 32) // 64 * 64)


def draw(rng):
    kind = rng.choice(["glu_fwd", "glu_fwd", "glu_bwd", "muon", "muon", "linear_i8", "linear_i8"])
    if kind == "muon":
        return {"kind": kind, "matrices": _log(rng, 1, 24), "longest": _log(rng, 32, 4096), "pick": rng.randrange(1 << 30),
                "grad": rng.choice(["f32", "f32", "bf16"])}
    few = rng.random() < 0.4  # a serving step
    if kind == "linear_i8":
        c, n = _features(rng, 64, 16384), _features(rng, 64, 32768)
        rows = _log(rng, 1, 32) if few else _log(rng, 16, max(16, min(16384, (1 << 38) // (c * n))))
        return {"kind": kind, "rows": rows, "c": c, "n": n, "out": rng.choice(["bf16", "bf16", "f32"])}
    c, f = _features(rng, 64, 8192), _features(rng, 64, 16384)
    rows = _log(rng, 1, 32) if few and kind == "glu_fwd" else _log(rng, 16, max(16, min(16384, (1 << 38) // (c * f))))
    case = {"kind": kind, "rows": rows, "c": c, "f": f, "act": rng.choice(["silu", "silu", "gelu", "relu"])}
    if kind == "glu_fwd":
        return {**case, "gu": rng.random() < 0.5}
    return {**case, "from": rng.choice(["gu", "x"])}


def _sides(case):
    if "model" in case:
        return MODELS[case["model"]]
    rng = random.Random(case["pick"])
    sides = [(_log(rng, 8, case["longest"]), _log(rng, 8, case["longest"])) for _ in range(case["matrices"])]
    return [(case["longest"], sides[0][1])] + sides[1:]


# ------------------------------------------------------------------------------------ inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _shifts(device):
    """Bit of the magnitude (the sign's is 8 higher) of element 2 j + h of a packed word, as [8][2]."""
    return (torch.arange(8, device=device)[:, None] + 16 * torch.arange(2, device=device)).to(torch.int32)


def _pack(two, neg):
    """Codes [k][n], k and n multiples of 64 -> the words of the packed layout: 64 filters x 64 elements a block."""
    k, n = two.shape
    sh = _shifts(two.device)
    # no two bits of a word meet, so that their sum, which wraps, is their union
    bits = (two.view(k // 64, 64, n // 64, 4, 8, 2).to(torch.int32) << sh) + (
        neg.view(k // 64, 64, n // 64, 4, 8, 2).to(torch.int32) << (sh + 8))
    return bits.sum((4, 5), dtype=torch.int32).permute(0, 2, 1, 3).contiguous().view(-1)


def _unpack(words, k, n):
    """The values of packed words: [k][n] fp32 of -2, -1, 1, 2."""
    kb, nb = -(-k // 64), -(-n // 64)
    w = words.view(kb, nb, 64, 4).permute(0, 2, 1, 3)[..., None, None]
    sh = _shifts(words.device)
    v = (1 + ((w >> sh) & 1)) * (1 - 2 * ((w >> (sh + 8)) & 1))
    return v.reshape(kb * 64, nb * 64)[:k, :n].float()


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, device=dev).normal_(mean, std, generator=g).to(dtype)

    kind = case["kind"]
    if kind in ("glu_fwd", "glu_bwd"):
        rows, c, f = case["rows"], case["c"], case["f"]
        state = {"case": case, "x": normal(rows, c, dtype=torch.bfloat16)}
        # the codes of real weights of deviation 1, padding zero
        kp, np_ = -(-2 * f // 64) * 64, -(-c // 64) * 64
        w = normal(kp, np_)
        real = (torch.arange(kp, device=dev) < 2 * f)[:, None] & (torch.arange(np_, device=dev) < c)
        state["codes"] = _pack((w.abs() > 1) & real, (w <= 0) & real)
        state["alpha"] = normal(2 * f, std=0.1, mean=0.8).abs() / math.sqrt(c)
        if kind == "glu_bwd":
            state["dh"] = normal(rows, f, std=0.1, dtype=torch.bfloat16)
            if case["from"] == "gu":
                state["gu"] = normal(rows, 2 * f, dtype=torch.bfloat16)
        return state
    if kind == "muon":
        sides = _sides(case)
        state = {"case": case, "w": [normal(r, c, std=c ** -0.5) for r, c in sides], "m": [], "g": []}
        for r, c in sides:
            # gradients as layers have them: a few strong directions over noise
            few = max(1, min(r, c) // 16)
            strong = normal(r, few) @ normal(few, c) * (0.02 / math.sqrt(few))
            state["g"].append((strong + normal(r, c, std=0.01)).to(TYPES[case["grad"]]))
            state["m"].append(strong * 5 + normal(r, c, std=0.03))
        return state
    rows, c, n = case["rows"], case["c"], case["n"]
    cp = -(-c // 16) * 16  # rows of 8-bit values are padded with zeros to a multiple of 16
    w = normal(n, c)
    top = w.abs().amax(1, keepdim=True)
    q = torch.zeros(n, cp, dtype=torch.int8, device=dev)
    q[:, :c] = torch.round(w * torch.div(torch.full_like(top, 127.0), top)).to(torch.int8)
    x = normal(rows, c)
    x[:, :: max(1, c // 5)] *= 8  # a few features are far larger than the others
    return {"case": case, "x": x.to(torch.bfloat16), "wq": q, "w_scale": top[:, 0] * (1 / 127) / math.sqrt(c), "bias": normal(n, std=0.1)}


# ------------------------------------------------------------------------------------ a pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"glu_fwd": _glu_fwd, "glu_bwd": _glu_bwd, "muon": _muon, "linear_i8": _linear_i8}[kind](state)


def _own(kind, s):
    import paper_1701_00485_amd as tbn

    case = s["case"]
    if kind == "glu_fwd":
        h, gu = tbn.glu_fwd(s["x"], s["codes"], s["alpha"], act=case["act"], want_gu=case["gu"])
        return (h, gu) if case["gu"] else h
    if kind == "glu_bwd":
        if case["from"] == "gu":
            return tbn.glu_bwd(s["dh"], gu=s["gu"], act=case["act"], want_h=True)
        return tbn.glu_bwd(s["dh"], x=s["x"], codes=s["codes"], alpha=s["alpha"], act=case["act"], want_h=True)
    if kind == "muon":
        return tbn.muon_step(s["w"], s["m"], s["g"], lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, eps=EPS, steps=STEPS)
    q, scale = tbn.quantize_rows_i8(s["x"])
    return tbn.matmul_i8(q, scale, s["wq"], s["w_scale"], bias=s["bias"], out_dtype=TYPES[case["out"]])


def _act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        on = (g > 0).float()
        return g * on, on
    if name == "gelu":
        phi = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-g))
    return g * s, s * (1 + g * (1 - s))


def _projections(s):
    case = s["case"]
    w = _unpack(s["codes"], 2 * case["f"], case["c"]) * s["alpha"][:, None]
    return s["x"].float() @ w.t()


def _glu_fwd(s):
    f = s["case"]["f"]
    gu = _projections(s)
    h = (_act(s["case"]["act"], gu[:, :f])[0] * gu[:, f:]).to(torch.bfloat16)
    return (h, gu.to(torch.bfloat16)) if s["case"]["gu"] else h


def _glu_bwd(s):
    f = s["case"]["f"]
    gu = s["gu"].float() if s["case"]["from"] == "gu" else _projections(s)
    a, slope = _act(s["case"]["act"], gu[:, :f])
    u, dh = gu[:, f:], s["dh"].float()
    return torch.cat([dh * u * slope, dh * a], 1).to(torch.bfloat16), (a * u).to(torch.bfloat16)


def _muon(s):
    for w, m, g in zip(s["w"], s["m"], s["g"]):
        g = g.float()
        m.copy_(MOMENTUM * m + g)
        x = g + MOMENTUM * m
        x = x / (x.square().sum().sqrt() + EPS)
        tall = x.shape[0] > x.shape[1]
        if tall:
            x = x.t()
        for _ in range(STEPS):
            a = x @ x.t()
            x = POLY[0] * x + (POLY[1] * a + POLY[2] * (a @ a)) @ x
        if tall:
            x = x.t()
        w.copy_(w - LR * DECAY * w - LR * math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * x)
    return s["w"], s["m"]


def _linear_i8(s):
    x = s["x"].float()
    top = x.abs().amax(1, keepdim=True)
    # two tensors divided, because a number over a tensor is its reciprocal times the number
    q = torch.round(x * torch.where(top > 0, torch.div(torch.full_like(top, 127.0), top), 0.0))
    y = (q @ s["wq"].float()[:, : s["case"]["c"]].t()) * ((top * (1 / 127)) * s["w_scale"]) + s["bias"]
    return y.to(TYPES[s["case"]["out"]])


# ------------------------------------------------------------------------------- what it costs
def work(case):
    kind = case["kind"]
    if kind in ("glu_fwd", "glu_bwd"):
        rows, c, f = case["rows"], case["c"], case["f"]
        weights = 2 * f * (c / 4 + 4)
        if kind == "glu_fwd":
            return {"bytes": int(weights + rows * (2 * c + 2 * f + (4 * f if case["gu"] else 0))), "flops": 4 * rows * c * f}
        if case["from"] == "gu":
            return {"bytes": rows * f * 12, "flops": 14 * rows * f}
        return {"bytes": int(weights + rows * (2 * c + 8 * f)), "flops": 4 * rows * c * f}
    if kind == "muon":
        size, b, fl = 2 if case["grad"] == "bf16" else 4, 0, 0
        for r, c in _sides(case):
            m, n = min(r, c), max(r, c)
            b += r * c * (16 + size)
            # a step: half of two symmetric products (m m n and m m m) and a whole one (m m n), two operations a term
            fl += STEPS * (m * m * n + m * m * m + 2 * m * m * n)
        return {"bytes": b, "flops": fl}
    rows, c, n = case["rows"], case["c"], case["n"]
    out = 2 if case["out"] == "bf16" else 4
    return {"bytes": rows * c * 2 + n * (c + 8) + rows * n * out, "flops": 2 * rows * c * n}


# ------------------------------------------------------------------------- results in 64 bits
def exact(case, seed):
    """What `run` returns for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    return {"glu_fwd": _exact_glu, "glu_bwd": _exact_glu, "muon": _exact_muon, "linear_i8": _exact_i8}[case["kind"]](case, s)


def _exact_codes(words, k, n):
    """Each code from its own word and bit."""
    i, kk = torch.arange(n, device=words.device), torch.arange(k, device=words.device)[:, None]
    nb = (n + 63) // 64
    word = words[((kk // 64 * nb + i // 64) * 64 + kk % 64) * 4 + i % 64 // 16].long()
    bit = 16 * (i % 2) + i % 16 // 2
    two, neg = word.bitwise_right_shift(bit).bitwise_and(1), word.bitwise_right_shift(bit + 8).bitwise_and(1)
    return torch.where(two.bool(), 2.0, 1.0).double() * torch.where(neg.bool(), -1.0, 1.0)


def _exact_glu(case, s):
    f = case["f"]
    if "gu" in s:
        gate, up = s["gu"].double().chunk(2, 1)
    else:
        x, alpha = s["x"].double(), s["alpha"].double()
        codes = _exact_codes(s["codes"], 2 * f, case["c"])
        gate, up = (x @ codes[:f].t()) * alpha[:f], (x @ codes[f:].t()) * alpha[f:]
    if case["act"] == "silu":
        t = torch.tanh(gate / 2)
        a, slope = gate * (1 + t) / 2, (1 + t) / 2 + gate * (1 - t * t) / 4
    elif case["act"] == "gelu":
        cdf = torch.special.erfc(-gate / math.sqrt(2)) / 2
        a, slope = gate * cdf, cdf + gate * (-(gate ** 2) / 2).exp() / math.sqrt(2 * math.pi)
    else:
        a, slope = gate.clamp(min=0), torch.heaviside(gate, torch.zeros_like(gate))
    if case["kind"] == "glu_fwd":
        return (a * up, torch.cat([gate, up], 1)) if case["gu"] else a * up
    dh = s["dh"].double()
    return torch.cat([slope * up * dh, a * dh], 1), a * up


def _exact_muon(case, s):
    """The polynomials act on the Gram matrix alone: X5 = P5 .. P1 X0 with Pk = p(Ak) and A(k+1) = Pk Ak Pk."""
    ws, ms = [], []
    for w, m, g in zip(s["w"], s["m"], s["g"]):
        w, m, g = w.double(), m.double(), g.double()
        m = torch.add(g, m, alpha=MOMENTUM)
        x = torch.add(g, m, alpha=MOMENTUM)
        x = x / (torch.linalg.vector_norm(x) + EPS)
        left = x.shape[0] <= x.shape[1]
        gram = x.mm(x.t()) if left else x.t().mm(x)
        eye = torch.eye(gram.shape[0], dtype=gram.dtype, device=gram.device)
        total = eye
        for _ in range(STEPS):
            p = torch.addmm(eye, gram, torch.add(eye * POLY[1], gram, alpha=POLY[2]), beta=POLY[0])
            total = p.mm(total)
            gram = p.mm(gram).mm(p)
        o = total.mm(x) if left else x.mm(total)
        ws.append((1 - LR * DECAY) * w - LR * max(1.0, w.shape[0] / w.shape[1]) ** 0.5 * o)
        ms.append(m)
    return ws, ms


def _exact_i8(case, s):
    """From the 8-bit values that the rounding gives: it is part of the definition, in 32 bits."""
    x = s["x"].float()
    top = torch.linalg.vector_norm(x, float("inf"), dim=1)
    q = torch.zeros_like(x)
    some = top > 0
    q[some] = (x[some] * torch.div(torch.full_like(top[some], 127.0), top[some])[:, None]).round().clamp(-127, 127)
    y = q.double().mm(s["wq"][:, : case["c"]].double().t())
    return torch.addcmul(s["bias"].double(), y, torch.outer(top.double() / 127, s["w_scale"].double()))
