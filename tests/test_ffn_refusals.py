"""What the gated block, Muon's step and the 8-bit products refuse, on the CPU: every call here fails its checks before
anything is launched (through the C ABI on addresses that are never followed, through Python on host tensors)."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_1701_00485_amd as tbn

GOOD, BAD = 0x10000000, 0x10000002
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
NAN, INF = float("nan"), float("inf")
# places that do not meet
P = [0x10000000 * k for k in range(1, 9)]


def _glu(rows=4, c=16, f=8, act=0):
    return tbn.GluDesc(rows, c, f, act)


def test_glu_sizes():
    lib, b = tbn.load(), ctypes.c_size_t()
    size = lambda d: lib.tbn_glu_workspace_size(ctypes.byref(d), ctypes.byref(b))  # noqa: E731
    for d in (_glu(rows=0), _glu(rows=-1), _glu(c=0), _glu(f=0), _glu(c=(1 << 20) + 1), _glu(f=(1 << 24) + 1), _glu(rows=(1 << 30) + 1),
              _glu(rows=1 << 30, c=16), _glu(rows=1 << 30, c=8, f=32), _glu(c=1 << 20, f=1 << 12)):
        assert size(d) == SHAPE, (d.rows, d.c, d.f)
    assert size(_glu(act=3)) == UNSUPPORTED and size(_glu(act=-1)) == UNSUPPORTED
    assert lib.tbn_glu_workspace_size(None, ctypes.byref(b)) == NULL
    assert lib.tbn_glu_workspace_size(ctypes.byref(_glu()), None) == NULL
    assert tbn.glu_workspace_size(_glu()) == 0
    # rows that are no multiple of 8 features are copied into padded ones
    assert tbn.glu_workspace_size(_glu(rows=5, c=13)) == 5 * 16 * 2


def test_glu_fwd():
    def fwd(desc=_glu(), x=P[0], codes=P[1], alpha=P[2], h=P[3], ht=0, gu=None, ws=None, size=0):
        return tbn.load().tbn_glu_fwd(desc and ctypes.byref(desc), x, codes, alpha, h, ht, gu, ws, size, None)

    assert fwd(desc=None) == fwd(x=None) == fwd(codes=None) == fwd(alpha=None) == fwd(h=None) == NULL
    assert fwd(desc=_glu(f=0)) == SHAPE and fwd(ht=2) == fwd(desc=_glu(act=9)) == UNSUPPORTED
    for name in ("x", "codes", "alpha", "h", "gu"):
        assert fwd(**{name: BAD}) == ALIGN, name
    odd = _glu(c=13)
    assert fwd(desc=odd) == WORKSPACE and fwd(desc=odd, ws=P[4], size=4 * 16 * 2 - 1) == WORKSPACE
    assert fwd(desc=odd, ws=BAD, size=4 * 16 * 2) == ALIGN
    # outputs over inputs, over each other, and the workspace over either: 4 x 16 of bf16, 1 KiB of codes, 4 x 8 and 4 x 16 of bf16
    for kw in ({"h": P[0]}, {"h": P[0] + 112}, {"h": P[1] + 1008}, {"h": P[2] + 48}, {"gu": P[0]}, {"gu": P[3]}, {"gu": P[3] - 112},
               {"desc": odd, "ws": P[3], "size": 128}, {"desc": odd, "ws": P[0], "size": 128}):
        assert fwd(**kw) == SHAPE, kw


def test_glu_bwd():
    def bwd(desc=_glu(), dh=P[0], gu=P[1], x=None, codes=None, alpha=None, dgu=P[2], h=None, ht=0, ws=None, size=0):
        return tbn.load().tbn_glu_bwd(desc and ctypes.byref(desc), dh, gu, x, codes, alpha, dgu, h, ht, ws, size, None)

    again = {"gu": None, "x": P[3], "codes": P[4], "alpha": P[5]}
    assert bwd(desc=None) == bwd(dh=None) == bwd(dgu=None) == NULL
    for name in ("x", "codes", "alpha"):
        assert bwd(**{**again, name: None}) == NULL and bwd(**{**again, name: BAD}) == ALIGN
    assert bwd(desc=_glu(rows=0)) == SHAPE and bwd(ht=5) == UNSUPPORTED
    for name in ("dh", "gu", "dgu", "h"):
        assert bwd(**{name: BAD}) == ALIGN, name
    odd = _glu(c=13)
    assert bwd(desc=odd, **again) == WORKSPACE and bwd(desc=odd, ws=P[6], size=127, **again) == WORKSPACE
    for kw in ({"dgu": P[0]}, {"dgu": P[1]}, {"h": P[0]}, {"h": P[1] + 112}, {"h": P[2] + 112}, {**again, "dgu": P[3]}, {**again, "h": P[4]},
               {**again, "h": P[5]}, {**again, "desc": odd, "ws": P[2], "size": 128}):
        assert bwd(**kw) == SHAPE, kw


def _muon(n=1, rows=8, cols=16, gt=1, w=P[0], m=P[1], g=P[2], ws=P[3], size=None, decay=0.0, scale=1.0, same=False, hyper=True, **h):
    lib = tbn.load()
    table = (tbn.MuonTensor * max(n, 1))()
    for i in range(n):
        off = 0 if same else i * 0x1000
        table[i] = tbn.MuonTensor(w and w + off, m and m + off, g, rows, cols, decay, scale)
    if size is None:
        b = ctypes.c_size_t()
        st = lib.tbn_muon_workspace_size(table, n, ctypes.byref(b))
        if st:
            return st
        size = b.value
    hy = tbn.MuonHyper(0.02, 0.95, 1e-7, 5, 1, None)
    for k, x in h.items():
        setattr(hy, k, x)
    return lib.tbn_muon_step(table, n, gt, ctypes.byref(hy) if hyper else None, ws, size, None)


def test_muon():
    lib, b = tbn.load(), ctypes.c_size_t()
    assert lib.tbn_muon_step(None, 1, 0, None, None, 0, None) == NULL
    assert lib.tbn_muon_workspace_size(None, 1, ctypes.byref(b)) == NULL
    assert lib.tbn_muon_workspace_size((tbn.MuonTensor * 1)(), 1, None) == NULL
    assert _muon(n=0) == SHAPE and _muon(rows=0) == SHAPE and _muon(cols=-1) == SHAPE
    assert _muon(rows=(1 << 20) + 1) == SHAPE and _muon(cols=(1 << 20) + 1) == SHAPE and _muon(rows=1 << 16, cols=1 << 15) == SHAPE
    assert _muon(w=None) == _muon(m=None) == _muon(g=None) == _muon(hyper=False) == NULL
    assert _muon(gt=2) == UNSUPPORTED
    assert _muon(w=P[0] + 2) == _muon(m=P[1] + 1) == _muon(g=P[2] + 2) == _muon(gt=0, g=P[2] + 1) == _muon(lr_dev=BAD) == ALIGN
    for k, bad in (("momentum", (1.0, 1.0 - 1e-9, -0.1, NAN)), ("eps", (0.0, 1e-31, 2.0, NAN)), ("steps", (0, -1, 33)), ("lr", (NAN, INF, 1e39))):
        assert all(_muon(**{k: v}) == SHAPE for v in bad), k
    assert _muon(decay=NAN) == _muon(scale=INF) == SHAPE
    assert _muon(ws=None) == _muon(size=1000) == WORKSPACE and _muon(ws=P[3] + 8) == ALIGN
    # a matrix twice, arrays that reach into each other, a gradient or the rate in what is written, the workspace over any of them
    assert _muon(n=2, same=True) == SHAPE and _muon(n=2, rows=80) == SHAPE
    assert _muon(m=P[0] + 508) == _muon(g=P[0] + 508) == _muon(g=P[1]) == _muon(ws=P[0]) == _muon(ws=P[2]) == SHAPE
    assert _muon(lr_dev=P[1] + 508) == _muon(lr_dev=P[3] + 64) == SHAPE


def test_rows_i8():
    def rows(x=P[0], xt=0, rows=4, c=20, q=P[1], scale=P[2]):
        return tbn.load().tbn_quantize_rows_i8(x, xt, rows, c, q, scale, None)

    assert rows(x=None) == rows(q=None) == rows(scale=None) == NULL
    assert rows(rows=0) == rows(c=0) == rows(rows=-4) == rows(c=(1 << 24) + 1) == rows(rows=(1 << 30) + 1) == rows(rows=1 << 30, c=17) == SHAPE
    assert rows(xt=2) == UNSUPPORTED
    assert rows(x=BAD) == rows(q=BAD) == rows(scale=BAD) == ALIGN
    # 4 x 20 of bf16 (160 bytes), 4 x 32 of int8, 4 scales
    assert rows(q=P[0] + 144) == rows(scale=P[0] + 156) == rows(scale=P[1] + 124) == SHAPE


def test_matmul_i8():
    def mul(rows=4, n=8, c=32, q=P[0], xs=P[1], w=P[2], ws=P[3], y=P[4], yt=0, ep=True, **e):
        p = tbn.Epilogue(None, None, None, 0)
        for k, v in e.items():
            setattr(p, k, v)
        return tbn.load().tbn_matmul_i8(rows, n, c, q, xs, w, ws, ctypes.byref(p) if ep else None, y, yt, None)

    assert mul(q=None) == mul(xs=None) == mul(w=None) == mul(ws=None) == mul(y=None) == NULL
    for kw in ({"rows": 0}, {"n": 0}, {"c": 0}, {"c": 24}, {"c": 131072}, {"n": (1 << 24) + 1}, {"rows": (1 << 30) + 1}, {"rows": 1 << 30},
               {"rows": 1 << 27, "n": 256}, {"n": 1 << 24, "c": 131056}):
        assert mul(**kw) == SHAPE, kw
    assert mul(yt=2) == UNSUPPORTED
    for kw in ({"q": BAD}, {"w": BAD}, {"xs": BAD}, {"ws": BAD}, {"y": BAD}, {"scale": BAD}, {"bias": BAD}, {"residual": BAD}):
        assert mul(**kw) == ALIGN, kw
    for kw in ({"y": P[0]}, {"y": P[2] + 240}, {"y": P[1]}, {"y": P[3] + 16}, {"bias": P[4] + 32}, {"scale": P[4] + 32},
               {"residual": P[4] + 16}):
        assert mul(**kw) == SHAPE, kw


def _zeros(*shape, t=torch.float32):
    return torch.zeros(shape, dtype=t)


BF, I32, I8 = torch.bfloat16, torch.int32, torch.int8


def test_python_sizes_and_types():
    x, codes, alpha, dh = _zeros(3, 16, t=BF), _zeros(256, t=I32), _zeros(8), _zeros(3, 4, t=BF)
    for kw, say in (({"codes": _zeros(255, t=I32)}, "codes has"), ({"alpha": _zeros(7)}, "alpha has"), ({"act": "tanh"}, "act is"),
                    ({"x": _zeros(0, 16, t=BF)}, "x has no")):
        with pytest.raises(ValueError, match=say):
            tbn.glu_fwd(**{**dict(x=x, codes=codes, alpha=alpha), **kw})
    for kw, say in (({"gu": _zeros(3, 7, t=BF)}, "gu has"), ({"x": x}, "needs gu"), ({"x": x, "codes": codes, "alpha": _zeros(6)}, "alpha has"),
                    ({"x": x[:2], "codes": codes, "alpha": alpha}, "x has 2 rows"), ({"gu": _zeros(3, 8, t=BF), "act": 1}, "act is")):
        with pytest.raises(ValueError, match=say):
            tbn.glu_bwd(dh, **kw)
    w, m, g = [_zeros(4, 6)], [_zeros(4, 6)], [_zeros(4, 6)]
    for kw, say in (({"w": []}, "no tensors"), ({"w": [_zeros(24)]}, "no matrix"), ({"m": [_zeros(4, 5)]}, r"m\[0\] has"), ({"g": g + g}, "g has 2"),
                    ({"scale": [1.0, 1.0]}, "scale has 2"), ({"weight_decay": []}, "weight_decay has 0"), ({"w": [_zeros(1, (1 << 20) + 1)]}, "side")):
        with pytest.raises(ValueError, match=say):
            tbn.muon_step(**{**dict(w=w, m=m, g=g), **kw})
    with pytest.raises(TypeError):
        tbn.muon_step(w, m, [_zeros(4, 6, t=torch.float16)])
    q, s, wq, ws = _zeros(3, 16, t=I8), _zeros(3), _zeros(5, 16, t=I8), _zeros(5)
    for kw, say in (({"wq": _zeros(5, 32, t=I8)}, "wq has rows"), ({"x_scale": _zeros(2)}, "x_scale has"), ({"w_scale": _zeros(4)}, "w_scale has"),
                    ({"bias": _zeros(4)}, "bias has"), ({"scale": _zeros(4)}, "scale has")):
        with pytest.raises(ValueError, match=say):
            tbn.matmul_i8(**{**dict(xq=q, x_scale=s, wq=wq, w_scale=ws), **kw})
    # host tensors and other types
    for call in (lambda: tbn.glu_fwd(x, codes, alpha), lambda: tbn.glu_bwd(dh, gu=_zeros(3, 8, t=BF)), lambda: tbn.muon_step(w, m, g),
                 lambda: tbn.quantize_rows_i8(x), lambda: tbn.matmul_i8(q, s, wq, ws)):
        with pytest.raises(TypeError, match="must be a CUDA"):
            call()


def test_muon_workspace_grows_with_its_matrices():
    small, large = [torch.empty(8, 8, device="meta")], [torch.empty(1000, 2000, device="meta")]
    a, b = tbn.muon_workspace_size(small), tbn.muon_workspace_size(large)
    assert 0 < a < b and b >= 4 * 1000 * 2000 * 4
    # many matrices share launches up to 64, and the workspace of one group
    assert tbn.muon_workspace_size(small * 200) == tbn.muon_workspace_size(small * 64)


# A step's tables take 34 words a matrix and 36 lists of its matrices, 1000 words a launch: one launch for 1 matrix, two for 20,
# more for 29 and up.
_WITHOUT_A_GPU = """
import ctypes, paper_1701_00485_amd as tbn
lib = tbn.load()
for n in (1, 20, 29, 40, 64, 200):
    t, b = (tbn.MuonTensor * n)(), ctypes.c_size_t()
    for i in range(n):
        t[i] = tbn.MuonTensor(0x10000000 + i * 0x1000, 0x20000000 + i * 0x1000, 0x30000000, 8, 16, 0.0, 1.0)
    h = tbn.MuonHyper(0.02, 0.95, 1e-7, 5, 1, None)
    assert lib.tbn_muon_workspace_size(t, n, ctypes.byref(b)) == 0
    print(n, lib.tbn_muon_step(t, n, 1, ctypes.byref(h), 0x40000000, b.value, None), lib.tbn_last_error().decode())
"""


@pytest.mark.skipif(torch.cuda.is_available(), reason="launches have to fail")
def test_muon_reports_a_launch_that_failed():
    """Without a GPU the first launch of a step fails: every length of list has that error, and the tables' other words go nowhere."""
    r = subprocess.run([sys.executable, "-c", _WITHOUT_A_GPU], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:]
    said = [line.split(" ", 2) for line in r.stdout.splitlines() if line.split(" ", 1)[0].isdigit()]
    assert [s[0] for s in said] == ["1", "20", "29", "40", "64", "200"]
    assert all(s[1] == "6" and s[2].startswith("tbn_muon_step: ") and s[2] == said[0][2] for s in said), said
