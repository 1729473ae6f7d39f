"""A mask's numbers are those of the calls that were made with it: they cannot be changed under a backward pass that is still to come."""
import pytest
import torch

import paper_2209_10778_b200 as nfad
from paper_2209_10778_b200 import block


@pytest.mark.parametrize("name,value", [("p", 0.25), ("seed", 9), ("offset", 8), ("step", None)])
def test_numbers_cannot_be_set(name, value):
    drop = nfad.Dropout(0.5, 7, 3)
    with pytest.raises(AttributeError):
        setattr(drop, name, value)
    assert (drop.p, drop.seed, drop.offset, drop.step) == (0.5, 7, 3, None)
    assert (drop.desc.p, drop.desc.seed, drop.desc.offset, drop.desc.step) == (0.5, 7, 3, None)
    with pytest.raises(AttributeError):
        drop.offset += 1


def test_the_step_is_read_where_it_is():
    # the argument check alone, on host tensors: the address that the library gets follows the tensor to another storage
    drop, x = nfad.Dropout(0.5, 7, 3), torch.zeros(4)
    drop._step = torch.zeros(1, dtype=torch.int64)
    for _ in range(2):
        block._mask(drop, x)
        assert drop.desc.step == drop.step.data_ptr()
        drop.step.data = torch.ones(1, dtype=torch.int64)
