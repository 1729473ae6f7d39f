"""A mask's numbers are those of the calls that were made with it: they cannot be changed under a backward pass that is still to come."""
import pytest

import paper_2209_10778_b200 as nfad


@pytest.mark.parametrize("name,value", [("p", 0.25), ("seed", 9), ("offset", 8), ("step", None)])
def test_numbers_cannot_be_set(name, value):
    drop = nfad.Dropout(0.5, 7, 3)
    with pytest.raises(AttributeError):
        setattr(drop, name, value)
    assert (drop.p, drop.seed, drop.offset, drop.step) == (0.5, 7, 3, None)
    assert (drop.desc.p, drop.desc.seed, drop.desc.offset, drop.desc.step) == (0.5, 7, 3, None)
    with pytest.raises(AttributeError):
        drop.offset += 1
