"""What the interface says of the precision of grouped-head attention, for each
kernel: sums and statistics of 32 bits, weights in as many bf16 parts as it names."""
import numpy as np
import pytest
import torch

from head_cases import HeadCase, random_tree
from head_ways import precise, run_way

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32

# Which kernel: requests, new tokens, heads, groups, form.
CALLS = {
    "few": dict(seq=[3000, 70, 501], new=[4, 2, 1], H=16, G=4, form="split"),
    "whole": dict(seq=[400, 70, 300], new=[200, 70, 1], H=8, G=2, form="whole"),
    "cut": dict(seq=[3000, 2500], new=[150, 61], H=16, G=1, form="split"),
    "cut-many": dict(seq=[2100, 1500], new=[300, 261], H=16, G=2, form="split"),
}


def _case(call, D, tree, seed):
    kw = dict(CALLS[call])
    form = kw.pop("form")
    if tree:
        kw["tree"] = random_tree(kw["new"], -(-max(kw["new"]) // 32), np.random.default_rng(seed))
    return HeadCase(D=D, seed=seed, **kw), form


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_lse_is_of_32_bits(D, y_dtype, tree, call):
    """A score sums D exact products in 32 bits: off by at most 128 half steps of scale * sum |q| |k| =: sa, and a few of
    its own, 2^-16 sa + 2^-20 in all; the sum of the weights is relatively off by as much, and of up to 3000 addends
    in eights and more that are added one after the other (a lane's, a few hundred at most) by 2^-15 at the worst of
    all roundings one way, 2^-20 as they fall; the logarithm and the maximum's product by a few half steps."""
    c, form = _case(call, D, tree, 40)
    (_, lse), way = run_way(c, DEV, form, y_dtype=y_dtype)
    assert way == call.split("-")[0]
    _, rl, _, sa = c.ref()
    none = np.isneginf(rl)
    assert np.array_equal(np.isneginf(lse), none)
    tol = (2.0 ** -16 * sa + 2.0 ** -19 + 2.0 ** -21 * np.abs(np.where(none, 0.0, rl)))[~none]
    off = np.abs(lse[~none] - rl[~none])
    assert np.all(off <= tol), (off / tol).max()


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("D", [64, 128])
def test_lse_does_not_change_the_result(D, call):
    c, form = _case(call, D, False, 41)
    (with_lse, _), _ = run_way(c, DEV, form)
    (without, _), _ = run_way(c, DEV, form, lse=False)
    assert np.array_equal(with_lse, without)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("y_dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_results_have_the_parts_of_their_weights(D, y_dtype, tree, call):
    """Three bf16 parts for 32-bit results; for bf16 results two in the kernel of few rows, one in that of many."""
    c, form = _case(call, D, tree, 42)
    (y, _), way = run_way(c, DEV, form, y_dtype=y_dtype)
    assert way == call.split("-")[0]
    assert precise(y, c.ref()[0], y_dtype, 3 if y_dtype == F32 else 2 if way == "few" else 1)
