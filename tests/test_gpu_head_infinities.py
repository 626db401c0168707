"""Infinities and NaNs of seen values where the parts of a row's tokens have
weights far apart: whichever wave, share or piece has them, they are in their
places of the result."""
import numpy as np
import pytest
import torch

from head_cases import HeadCase, chain_tree, check_heads
from head_ways import run_way

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32
PLACES = ((2, float("inf")), (17, float("nan")), (63, -float("inf")))


def _peaked(seq, new, peak, odd, tree=None, **kw):
    """All queries are ones, and one token's key is 16 in all places: its score is 2^130 and more times the others' in
    weight, so that every part of the tokens without it counts nothing.  The values of tokens `odd` hold no numbers."""
    c = HeadCase(seq=[seq], new=[new], tree=tree, **kw)
    c.q.fill_(1.0)
    c.put(0, peak, k=torch.full((c.G, c.D), 16.0, dtype=BF))
    clean = [c.v[0][at].clone() for at in odd]
    for at, v in zip(odd, clean):
        bad = v.clone()
        for d, x in PLACES:
            bad[:, d] = x
        c.put(0, at, v=bad)
    return c, clean


def _check(c, clean, odd, got, y_dtype):
    for at, v in zip(odd, clean):
        v[:, [d for d, _ in PLACES]] = 0.0
        c.put(0, at, v=v)
    ry, rl, ya, sa = c.ref()
    y, lse = got
    for d, x in PLACES:
        assert np.array_equal(y[:, :, d], np.full_like(y[:, :, d], x), equal_nan=True), d
    keep = [d for d in range(c.D) if d not in [d for d, _ in PLACES]]
    # the peak's own score is far larger than what a weight may be off by, which is then nothing: it has all of it
    sa = np.minimum(sa, 16.0)
    check_heads((y[:, :, keep], lse), (ry[:, :, keep], rl, ya[:, :, keep], sa), y_dtype)


@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("peak,odd", [(5, [40]), (40, [5]), (5, [2990]), (2990, [3]), (1500, [70, 1400, 2900])])
@pytest.mark.parametrize("kind", ["few", "tree", "many", "whole"])
def test_a_part_without_weight_keeps_its_infinities(kind, peak, odd, D, y_dtype):
    """Another wave of one share, another share, another piece of a row tile, another tile of a whole one."""
    new = 9 if kind in ("few", "tree") else 250
    H, G = (16, 2) if kind in ("few", "tree") else (16, 1)
    c, clean = _peaked(3001 + new, new, peak, odd, tree=chain_tree([new], 1) if kind == "tree" else None, H=H, G=G, D=D,
                       seed=len(odd))
    got, way = run_way(c, DEV, "whole" if kind == "whole" else "split", y_dtype=y_dtype)
    assert way == dict(few="few", tree="few", many="cut", whole="whole")[kind]
    _check(c, clean, odd, got, y_dtype)


@pytest.mark.parametrize("new,heads", [(1, 4), (2, 64), (40, 128)])
@pytest.mark.parametrize("y_dtype", [BF, F32])
def test_a_short_list_keeps_them_too(y_dtype, new, heads):
    """One share, whose waves meet in the workgroup, in either form."""
    for form in ("split", "whole"):
        c, clean = _peaked(100 + new, new, 3, [60], H=heads, G=2, seed=3)
        got, _ = run_way(c, DEV, form, y_dtype=y_dtype)
        _check(c, clean, [60], got, y_dtype)


@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("seq,new,form,way", [(40, 2, "split", "few"), (40, 2, "whole", "whole"), (3000, 4, "split", "few"),
                                              (3000, 200, "split", "cut"), (3000, 200, "whole", "whole")])
def test_rows_of_no_weight_at_all(seq, new, form, way, y_dtype):
    """Every key's score is -inf: no weight is left, and the rows are zero but for the infinities of the values."""
    c = HeadCase(seq=[seq], new=[new], H=16, G=1, seed=4)
    c.q.fill_(1.0)
    for j in range(seq):
        k = c.k[0][j].clone()
        k[:, 0] = -float("inf")
        v = c.v[0][j].clone()
        if j % 37 == 5:
            v[:, 2], v[:, 17] = float("inf"), float("nan")
        c.put(0, j, k=k, v=v)
    (y, lse), ran = run_way(c, DEV, form, y_dtype=y_dtype)
    assert ran == way
    want = np.zeros_like(y)
    want[:, :, 2], want[:, :, 17] = np.inf, np.nan
    assert np.array_equal(y, want, equal_nan=True)
    assert np.all(np.isneginf(lse))
