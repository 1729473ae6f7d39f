"""The plain mask against the generator's published test vectors, and what a mask has to be."""
import numpy as np
import pytest

import dropout_plain as plain

VECTORS = [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
]


@pytest.mark.parametrize("counter,key,want", VECTORS)
def test_published_vectors(counter, key, want):
    got = plain.philox([np.array([c]) for c in counter], key)
    assert tuple(int(v[0]) for v in got) == want


def test_counter_words():
    # element 8 (2^32 + 3) + 5 of a call: the index's words, then offset's
    i, at, seed = 2 ** 32 + 3, (7 << 32) + 9, (5 << 32) + 11
    w = plain.philox([np.array([v]) for v in (3, 1, 9, 7)], (11, 5))
    assert plain.bits16(8, seed, at, 8 * i)[5] == int(w[2][0]) >> 16


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_share_and_independence(p):
    n = 1 << 20
    keep, scale = plain.mask(n, p, 1234567, 5)
    # six standard deviations of a binomial share
    assert abs(keep.double().mean().item() - (1 - np.rint(p * 65536) / 65536)) <= 6 * (p * (1 - p) / n) ** 0.5
    assert scale == 0 if p == 1.0 else abs(scale * (1 - p) - 1) < 2.0 ** -16 * scale
    if 0 < p < 1:
        other, _ = plain.mask(n, p, 1234567, 6)
        both = (keep & other).double().mean().item()
        assert abs(both - (1 - p) ** 2) <= 6 * (1 / n) ** 0.5 + 2.0 ** -15
