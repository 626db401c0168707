"""The checks of grouped heads' precision see what they are there for: weights
of a part less than the kernels say they have.  No GPU."""
import pytest
import torch

from head_ways import HeadCase, precise, with_weight_parts

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("seq,new", [(600, 3), (70, 40)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("y_dtype,parts", [(F32, 3), (BF, 2)])
def test_a_part_less_is_seen(y_dtype, parts, D, seq, new):
    c = HeadCase(seq=[seq], new=[new], H=8, G=2, D=D, seed=50)
    ref = c.ref()[0]
    assert precise(with_weight_parts(c, parts, y_dtype), ref, y_dtype, parts)
    assert not precise(with_weight_parts(c, parts - 1, y_dtype), ref, y_dtype, parts)


@pytest.mark.parametrize("D", [64, 128])
def test_one_part_is_within_its_own_bound(D):
    c = HeadCase(seq=[500], new=[60], H=8, G=2, D=D, seed=51)
    assert precise(with_weight_parts(c, 1, BF), c.ref()[0], BF, 1)
