"""The operators of fine-tuning and serving a frozen two-bit network, as cases to time and to compare:
layer norm (forward, backward), AdamW over many tensors (states in 32 or 8 bits) and the low-rank
adapters of many requests beside a shared projection (forward, backward).

`run` computes them in their plain form, elementary torch operations in 32 bits, or, where `own` is true, by the
calls of ``paper_1701_00485_amd``.  `exact` says what the definitions give in 64 bits.

Kinds of case (field "kind"):
  ln_fwd, ln_bwd            rows x c, x and y in "bf16" or "f32"
  adamw                     the tensors of a network of this repository ("model"), or `tensors` of them whose sizes are
                            drawn up to `largest` from `pick`; states in `bits` bits, gradients in "f32" or "bf16".
                            They lie in flat buffers, each beginning at a multiple of 256 elements
  adapter_fwd, adapter_bwd  rows of c features, k outputs, `bank` adapters of this rank held in "bf16" or "f32", the rows
                            those of `requests` requests of ragged lengths (as many as rows: one token each)
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-5
LR, B1, B2, ADAM_EPS, WD, SEED = 1e-3, 0.9, 0.999, 1e-8, 0.01, 7
BLOCK = 256  # elements that share a scale of an 8-bit state
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _resnet18():
    shapes, cin = [64 * 147], 64
    for cout in (64, 128, 256, 512):
        for block in range(2):
            shapes += [cout * 9 * cin, cout * 9 * cout] + ([cout * cin] if block == 0 and cin != cout else [])
            shapes += [cout] * (6 if block == 0 and cin != cout else 4)
            cin = cout
    return shapes + [64, 64, 1000 * 512, 1000]


MODELS = {
    "lenet": [32 * 25, 64 * 800, 512 * 3136, 10 * 512],
    "resnet18": _resnet18(),
    "fc": [32768 * 8192, 32768, 8192, 8192],  # a fully-connected layer 8192 -> 32768, its bias, a layer norm
}


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the smallest call: one token of a 512-feature network at inference, launch latency counts
        {"name": "ln_fwd_1x512", "kind": "ln_fwd", "rows": 1, "c": 512, "x": "bf16", "y": "bf16"},
        # a large batch in front of the 8192 -> 32768 layer
        {"name": "ln_fwd_8192x8192", "kind": "ln_fwd", "rows": 8192, "c": 8192, "x": "bf16", "y": "bf16"},
        # a ragged batch over 1000 features, the residual stream kept in 32 bits
        {"name": "ln_bwd_777x1000", "kind": "ln_bwd", "rows": 777, "c": 1000, "x": "f32", "y": "bf16"},
        # a large training batch
        {"name": "ln_bwd_16384x4096", "kind": "ln_bwd", "rows": 16384, "c": 4096, "x": "bf16", "y": "bf16"},
        # the four layers of LeNet: a small model's step
        {"name": "adamw32_lenet", "kind": "adamw", "model": "lenet", "bits": 32, "grad": "f32"},
        # the 62 tensors of ResNet-18, many of them of a few hundred elements
        {"name": "adamw8_resnet18", "kind": "adamw", "model": "resnet18", "bits": 8, "grad": "f32"},
        # a large fully-connected layer, states in 32 bits
        {"name": "adamw32_fc", "kind": "adamw", "model": "fc", "bits": 32, "grad": "f32"},
        # ... and in 8, with gradients that a backward pass left in 16
        {"name": "adamw8_fc", "kind": "adamw", "model": "fc", "bits": 8, "grad": "bf16"},
        # a serving step: one token of each of 48 requests beside the 8192 -> 32768 layer, adapters of their own
        {"name": "adapter_fwd_decode48", "kind": "adapter_fwd", "rows": 48, "c": 8192, "k": 32768, "rank": 16, "bank": 64,
         "weights": "bf16", "requests": 48, "out": "bf16"},
        # a batch of prompts of ragged lengths
        {"name": "adapter_fwd_5000", "kind": "adapter_fwd", "rows": 5000, "c": 4096, "k": 4096, "rank": 32, "bank": 8,
         "weights": "bf16", "requests": 11, "out": "bf16"},
        # fine-tuning the classifier of a 512-feature network, one adapter, a small batch
        {"name": "adapter_bwd_100", "kind": "adapter_bwd", "rows": 100, "c": 512, "k": 1000, "rank": 8, "bank": 1,
         "weights": "f32", "requests": 1, "out": "bf16"},
        # fine-tuning four adapters at once on long sequences, master weights in 32 bits
        {"name": "adapter_bwd_8192", "kind": "adapter_bwd", "rows": 8192, "c": 4096, "k": 8192, "rank": 16, "bank": 4,
         "weights": "f32", "requests": 8, "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """Mostly multiples of 64, as networks have; one in four as it falls."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.25 else max(64, (c + 32) // 64 * 64)


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_bwd", "adamw", "adamw", "adapter_fwd", "adapter_fwd", "adapter_bwd"])
    if kind in ("ln_fwd", "ln_bwd"):
        c = _features(rng, 16, 32768)
        return {"kind": kind, "rows": _log(rng, 1, max(1, (1 << 26) // c)), "c": c, "x": rng.choice(["bf16", "bf16", "f32"]),
                "y": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "adamw":
        return {"kind": kind, "tensors": _log(rng, 1, 200), "largest": _log(rng, 100, 1 << 24), "pick": rng.randrange(1 << 30),
                "bits": rng.choice([32, 8]), "grad": rng.choice(["f32", "f32", "bf16"])}
    c, k = _features(rng, 64, 8192), _features(rng, 64, 16384)
    rank = rng.choice([1, 4, 8, 8, 16, 16, 32, 64, 128, rng.randint(1, 128)])
    if kind == "adapter_fwd" and rng.random() < 0.6:
        rows = _log(rng, 1, 256)
        return {"kind": kind, "rows": rows, "c": c, "k": k, "rank": rank, "bank": _log(rng, 1, 64), "weights": "bf16",
                "requests": rows, "out": rng.choice(["bf16", "f32"])}
    rows = _log(rng, 16, 8192 if kind == "adapter_fwd" else 4096)
    return {"kind": kind, "rows": rows, "c": c, "k": k, "rank": rank, "bank": _log(rng, 1, 8),
            "weights": rng.choice(["f32", "bf16"]), "requests": min(rows, _log(rng, 1, 24)), "out": rng.choice(["bf16", "bf16", "f32"])}


def _sizes(case):
    if "model" in case:
        return MODELS[case["model"]]
    rng = random.Random(case["pick"])
    return [case["largest"]] + [_log(rng, 1, case["largest"]) for _ in range(case["tensors"] - 1)]


# ------------------------------------------------------------------------------------ inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _rows_of_requests(case, seed):
    """The adapter of each row: requests of ragged lengths, one in twelve without an adapter (-1)."""
    rng = random.Random(seed)
    n, rows = case["requests"], case["rows"]
    cuts = list(range(rows + 1)) if n == rows else [0] + sorted(rng.sample(range(1, rows), n - 1)) + [rows]
    ids = [-1 if n > 1 and rng.random() < 1 / 12 else rng.randrange(case["bank"]) for _ in range(n)]
    return [a for a, lo, hi in zip(ids, cuts, cuts[1:]) for _ in range(hi - lo)]


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.empty(shape, device=dev).normal_(mean, std, generator=g).to(dtype)

    kind = case["kind"]
    if kind in ("ln_fwd", "ln_bwd"):
        rows, c, xt, yt = case["rows"], case["c"], TYPES[case["x"]], TYPES[case["y"]]
        x = normal(rows, c, std=1.5, mean=0.3, dtype=xt)
        gamma, beta = normal(c, std=0.2, mean=1.0), normal(c, std=0.1)
        if kind == "ln_fwd":
            return {"case": case, "x": x, "gamma": gamma, "beta": beta}
        mean = x.float().mean(1)
        inv_std = 1 / torch.sqrt((x.float() - mean[:, None]).square().mean(1) + EPS)
        return {"case": case, "x": x, "dy": normal(rows, c, std=0.01, dtype=yt), "mean": mean, "inv_std": inv_std, "gamma": gamma}
    if kind == "adamw":
        return _prepare_adamw(case, dev, normal)
    rows, c, k, r, bank = (case[f] for f in ("rows", "c", "k", "rank", "bank"))
    wt, ot = TYPES[case["weights"]], TYPES[case["out"]]
    state = {"case": case, "index": torch.tensor(_rows_of_requests(case, seed), dtype=torch.int32).to(dev),
             "x": normal(rows, c, dtype=torch.bfloat16), "a": normal(bank, r, c, std=c ** -0.5, dtype=wt),
             "b": normal(bank, k, r, std=0.5 * r ** -0.5, dtype=wt), "scale": normal(bank, std=0.1, mean=1.0).abs()}
    if kind == "adapter_fwd":
        state["residual"] = normal(rows, k, dtype=ot)
    else:
        state["dy"] = normal(rows, k, std=0.1, dtype=torch.bfloat16)
        state["residual"] = normal(rows, c, std=0.1, dtype=ot)
        state["t"] = _masked(state["x"].float() @ state["a"].float().flatten(0, 1).t(), state).sum(1)
    return state


def _prepare_adamw(case, dev, normal):
    """The state after some steps: parameters, gradients and moments in flat buffers, the tensors views of them."""
    sizes, bits = _sizes(case), case["bits"]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    w, g, m, v = normal(at, std=0.5), normal(at, std=0.01), normal(at, std=0.003), normal(at, std=0.01).square() + 1e-7
    live = torch.zeros(at, dtype=torch.bool, device=dev)
    for s, n in zip(starts, sizes):
        live[s:s + n] = True
    for t in (w, g, m, v):
        t.mul_(live)
    state = {"case": case, "sizes": sizes, "starts": starts, "w": w, "g": g.to(TYPES[case["grad"]]), "step": 100,
             "wd": [WD if n > 4096 else 0.0 for n in sizes]}
    if bits == 32:
        state.update(m=m, v=v)
    else:
        state["m_scale"], state["v_scale"] = (t.view(-1, BLOCK).abs().amax(1) / 448 for t in (m, v.sqrt()))
        for name, t in (("m", m), ("v", v.sqrt())):
            s = state[name + "_scale"][:, None]
            state[name] = torch.where(s > 0, t.view(-1, BLOCK) / s, 0.0).view(-1).to(torch.float8_e4m3fn)
    # what the program hands to the step: lists of tensors
    cut = lambda t: [t[s:s + n] for s, n in zip(starts, sizes)]  # noqa: E731
    state["lists"] = {f: cut(state[f]) for f in ("w", "m", "v", "g")}
    if bits == 8:
        for f in ("m_scale", "v_scale"):
            state["lists"][f] = [state[f][s // BLOCK:s // BLOCK - (-n // BLOCK)] for s, n in zip(starts, sizes)]
    return state


# ------------------------------------------------------------------------------------ a pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"ln_fwd": _ln_fwd, "ln_bwd": _ln_bwd, "adamw": _adamw, "adapter_fwd": _adapter_fwd, "adapter_bwd": _adapter_bwd}[kind](state)


def _own(kind, s):
    import paper_1701_00485_amd as tbn

    if kind == "ln_fwd":
        return tbn.layernorm_fwd(s["x"], s["gamma"], s["beta"], eps=EPS, out_dtype=TYPES[s["case"]["y"]])
    if kind == "ln_bwd":
        return tbn.layernorm_bwd(s["x"], s["dy"], s["mean"], s["inv_std"], s["gamma"])
    if kind == "adapter_fwd":
        return tbn.adapter_fwd(s["x"], s["index"], s["a"], s["b"], scale=s["scale"], residual=s["residual"])
    if kind == "adapter_bwd":
        return tbn.adapter_bwd(s["x"], s["dy"], s["index"], s["a"], s["b"], s["t"], scale=s["scale"], residual=s["residual"])
    l = s["lists"]
    more = {} if s["case"]["bits"] == 32 else {"m_scale": l["m_scale"], "v_scale": l["v_scale"], "seed": SEED}
    tbn.adamw_step(l["w"], l["m"], l["v"], l["g"], s["step"], lr=LR, beta1=B1, beta2=B2, eps=ADAM_EPS, weight_decay=s["wd"], **more)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    if s["case"]["bits"] == 32:
        return s["w"], s["m"], s["v"]
    return s["w"], s["m"], s["v"], s["m_scale"], s["v_scale"]


def _ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    inv_std = 1 / torch.sqrt((d * d).mean(1) + EPS)
    y = d * inv_std[:, None] * s["gamma"] + s["beta"]
    return y.to(TYPES[s["case"]["y"]]), mean, inv_std


def _ln_bwd(s):
    xh = (s["x"].float() - s["mean"][:, None]) * s["inv_std"][:, None]
    dy = s["dy"].float()
    h = dy * s["gamma"]
    dx = s["inv_std"][:, None] * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)


def _masked(t_all, s):
    """[rows][bank * rank] -> [rows][bank][rank], zero but for each row's own adapter."""
    bank = s["case"]["bank"]
    mine = s["index"][:, None] == torch.arange(bank, device=s["index"].device, dtype=torch.int32)
    return torch.where(mine[:, :, None], t_all.view(-1, bank, s["case"]["rank"]), 0.0)


def _adapter_fwd(s):
    a, b = s["a"].float(), s["b"].float()
    t = _masked(s["x"].float() @ a.flatten(0, 1).t(), s)
    y = (t * s["scale"][:, None]).flatten(1) @ b.transpose(1, 2).flatten(0, 1) + s["residual"].float()
    return y.to(s["residual"].dtype), t.sum(1)


def _adapter_bwd(s):
    a, b, x, dy = (s[f].float() for f in ("a", "b", "x", "dy"))
    dt = _masked(dy @ b.transpose(1, 2).flatten(0, 1).t(), s) * s["scale"][:, None]
    dx = dt.flatten(1) @ a.flatten(0, 1) + s["residual"].float()
    bank, rank = s["case"]["bank"], s["case"]["rank"]
    ts = _masked(s["t"].repeat(1, bank), s) * s["scale"][:, None]
    da = (dt.flatten(1).t() @ x).view(bank, rank, -1)
    db = (ts.flatten(1).t() @ dy).view(bank, rank, -1).transpose(1, 2).contiguous()
    return dx.to(s["residual"].dtype), da, db


def _mix(h):
    """A mixed 32-bit value of a 32-bit one (in int64)."""
    h = h & 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x9E3779B1) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _tensors(s):
    """Of every 256 elements of the flat buffers: their tensor, and where in it they begin."""
    dev = s["w"].device
    begins = torch.arange(0, s["w"].numel(), BLOCK, device=dev)
    starts = torch.tensor(s["starts"], device=dev)
    of = torch.searchsorted(starts, begins, right=True) - 1
    return of, begins - starts[of]


def _bits(s, of, begins):
    """32 random bits of every element: a function of seed, step, tensor and place in the tensor."""
    key = torch.tensor([_mix(_mix(_mix(SEED) ^ s["step"]) ^ i) for i in range(len(s["sizes"]))], device=of.device)
    place = begins[:, None] + torch.arange(BLOCK, device=of.device)
    return _mix(place ^ key[of][:, None]).view(-1)


def _codes(x, bits):
    """x / scale as E4M3 codes and the scales, a scale for every 256 values; rounded up with the probability `bits` / 2^20."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    u = torch.where(top > 0, x * (448 / top), 0.0).view(-1)
    a = u.abs()
    low = a < 2.0 ** -6  # below the smallest normal code the steps stay 2^-9
    a = torch.where(low, a + 2.0 ** -6, a)
    a = (((a.view(torch.int32) + bits) >> 20) << 20).view(torch.float32)
    a = torch.where(low, a - 2.0 ** -6, a)
    return torch.copysign(a.clamp(max=448.0), u).to(torch.float8_e4m3fn), top.view(-1) / 448


def _adamw(s):
    w, g, eight = s["w"], s["g"].float(), s["case"]["bits"] == 8
    of, begins = _tensors(s)
    wd = torch.tensor(s["wd"], device=w.device)[of][:, None].expand(-1, BLOCK).reshape(-1)
    if eight:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * (g * g)
    root = torch.sqrt(v)
    w.copy_(w - (LR * wd) * w - (LR / (1 - B1 ** s["step"])) * m / (root / math.sqrt(1 - B2 ** s["step"]) + ADAM_EPS))
    if eight:
        bits = _bits(s, of, begins)
        for name, x, b in (("m", m, bits & 0xFFFFF), ("v", root, bits >> 12)):
            codes, scale = _codes(x, b.to(torch.int32))
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_outputs(s)


# ------------------------------------------------------------------------------- what it costs
def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2}
    if kind in ("ln_fwd", "ln_bwd"):
        n, c, x, y = case["rows"] * case["c"], case["c"], size[case["x"]], size[case["y"]]
        if kind == "ln_fwd":
            return {"bytes": n * (x + y) + 8 * c + 8 * case["rows"], "flops": 8 * n}
        return {"bytes": n * (2 * x + y) + 12 * c + 8 * case["rows"], "flops": 14 * n}
    if kind == "adamw":
        n = sum(_sizes(case))
        states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (8 + size[case["grad"]] + states), "flops": 16 * n}
    rows, c, k, r = (case[f] for f in ("rows", "c", "k", "rank"))
    used = min(case["bank"], case["requests"])
    weights = used * r * (c + k) * size[case["weights"]]
    if kind == "adapter_fwd":
        return {"bytes": weights + rows * (2 * c + 4 * r + 4) + rows * k * 2 * size[case["out"]], "flops": 2 * rows * r * (c + k)}
    grads = case["bank"] * r * (c + k) * 4
    return {"bytes": weights + grads + rows * (2 * c + 2 * k + 4 * r + 4) + rows * c * 2 * size[case["out"]],
            "flops": 4 * rows * r * (c + k)}


# ------------------------------------------------------------------------- results in 64 bits
def exact(case, seed):
    """What `run` returns for these inputs, from the definitions in 64 bits.  A code of an 8-bit state has the value that
    its random rounding stands for: the moment over its scale."""
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    kind = case["kind"]
    if kind == "ln_fwd":
        mean = d["x"].sum(1) / case["c"]
        var = (d["x"] - mean[:, None]).pow(2).sum(1) / case["c"]
        xh = (d["x"] - mean[:, None]) * (var + EPS).rsqrt()[:, None]
        return torch.addcmul(d["beta"], xh, d["gamma"]), mean, (var + EPS).rsqrt()
    if kind == "ln_bwd":
        # the Jacobian of a row, applied to h: s (I - 1 1^T / c - xh xh^T / c) h
        xh = torch.addcmul(-(d["mean"] * d["inv_std"])[:, None], d["x"], d["inv_std"][:, None])
        h = d["dy"] * d["gamma"]
        along = torch.stack([h.sum(1), torch.linalg.vecdot(h, xh)]) / case["c"]
        dx = d["inv_std"][:, None] * torch.addcmul(h - along[0][:, None], xh, along[1][:, None], value=-1)
        return dx, torch.linalg.vecdot(d["dy"], xh, dim=0), torch.ones_like(d["mean"]) @ d["dy"]
    if kind == "adamw":
        return _exact_adamw(case, s, d)
    a, b, x = d["a"], d["b"], d["x"]
    index = s["index"].long()
    if kind == "adapter_fwd":
        y, t = d["residual"].clone(), x.new_zeros(case["rows"], case["rank"])
        for i in range(case["bank"]):
            at = torch.nonzero(index == i)[:, 0]
            t[at] = x[at] @ a[i].t()
            y[at] += d["scale"][i] * (t[at] @ b[i].t())
        return y, t
    dx, da, db = d["residual"].clone(), torch.zeros_like(a), torch.zeros_like(b)
    for i in range(case["bank"]):
        at = torch.nonzero(index == i)[:, 0]
        dt = d["scale"][i] * (d["dy"][at] @ b[i])
        dx[at] += dt @ a[i]
        da[i] = dt.t() @ x[at]
        db[i] = d["scale"][i] * (d["dy"][at].t() @ d["t"][at])
    return dx, da, db


def _exact_adamw(case, s, d):
    eight = case["bits"] == 8
    out = [torch.zeros_like(d["w"]) for _ in range(3)]
    scales = [torch.zeros_like(d["m_scale"]) for _ in range(2)] if eight else []
    for start, n, wd in zip(s["starts"], s["sizes"], s["wd"]):
        at = slice(start, start + n)
        g, m, v, w = d["g"][at], d["m"][at], d["v"][at], d["w"][at]
        if eight:
            of = torch.arange(start, start + n, device=g.device) // BLOCK
            m, v = m * d["m_scale"][of], (v * d["v_scale"][of]) ** 2
        m = torch.lerp(g, m, B1)
        v = torch.lerp(g ** 2, v, B2)
        step = (m / (1 - B1 ** s["step"])) / ((v / (1 - B2 ** s["step"])).sqrt() + ADAM_EPS)
        out[0][at] = w * (1 - LR * wd) - LR * step
        for x, o, k in ((m, out[1], 0), (v.sqrt() if eight else v, out[2], 1)):
            if eight:
                top = torch.zeros_like(scales[k]).scatter_reduce_(0, of, x.abs(), "amax")
                scales[k] += top / 448
                o[at] = x / (top[of] / 448)
            else:
                o[at] = x
    return tuple(out + scales)
