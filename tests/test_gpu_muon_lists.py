"""Muon's step over lists of matrices whose launches divide the stages of tiles over blocks: where a divided tile belongs to a matrix behind the
first, where a block's stages cross from one matrix into the next, and where matrices before have a block for every tile.  Each matrix against
64 bits, with the tolerances of test_gpu_muon.py.
"""
import pytest
import torch

from test_gpu_muon import BF, F, check

pytestmark = pytest.mark.gpu

LISTS = {
    # X X^T: few tiles, long rows; four matrices, blocks that cross between them
    "lenet": [(32, 25), (64, 800), (512, 3136), (10, 512)],
    # the products of a matrix's own polynomials, one large among small ones
    "one large": [(1276, 97), (96, 1339), (1584, 1438), (47, 1569), (1157, 83), (128, 476), (546, 620), (886, 167)],
    # ... and with tiles that have blocks of their own before the divided ones
    "large": [(1809, 925), (1405, 1351), (342, 532), (1901, 1864), (1023, 1792)],
    # the products with X, their last tiles: of the last matrix alone, of the last two, of the last four
    "equal": [(1024, 3000)] * 6,
    "wide and tall": [(259, 881), (282, 896), (1413, 434), (1060, 1248), (1253, 223), (1058, 171), (391, 392)],
    "square": [(1928, 1987), (1929, 1353), (274, 1104), (1536, 1415), (809, 1132), (57, 1051), (240, 227)],
}


def lists_of(sides, dtype, odd):
    """w, m and g side by side in one buffer each, every other matrix at a place that is no multiple of 16 bytes where `odd`."""
    g = torch.Generator(device="cuda").manual_seed(5)
    step = [r * c + (1 if odd else -r * c % 8) for r, c in sides]
    flat = [torch.empty(sum(step), device="cuda").normal_(std=s, generator=g).to(t) for s, t in ((1.0, F), (2.0, F), (1.0, dtype))]
    lists, at = [[], [], []], 0
    for (r, c), n in zip(sides, step):
        for l, f in zip(lists, flat):
            l.append(f[at:at + r * c].view(r, c))
        at += n
    return lists


@pytest.mark.parametrize("dtype,odd", [(F, False), (BF, False), (F, True), (BF, True)])
@pytest.mark.parametrize("name", LISTS)
def test_divided_launches_of_many_matrices(tbn, name, dtype, odd):
    lists = lists_of(LISTS[name], dtype, odd)
    w0, m0 = ([t.clone() for t in l] for l in lists[:2])
    decays = [0.01 * (i % 3) for i in range(len(w0))]
    tbn.muon_step(*lists, lr=0.5, weight_decay=decays)
    for i in range(len(w0)):
        check(lists[0][i], lists[1][i], w0[i], m0[i], lists[2][i], 0.5, wd=decays[i])
    first = [t.clone() for l in lists[:2] for t in l]
    for t, old in zip(lists[0] + lists[1], w0 + m0):
        t.copy_(old)
    tbn.muon_step(*lists, lr=0.5, weight_decay=decays)
    assert all(torch.equal(t, old) for t, old in zip(lists[0] + lists[1], first))
