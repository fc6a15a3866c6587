"""The dropout oracle against what does not come from it: the generator's published answers, its uniformity, and the
binomial law of the mask."""
import numpy as np
import pytest

from oracle import dropout as D


@pytest.mark.parametrize("counter,key,words", [      # the known answers its authors publish with the generator
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, words):
    assert tuple(int(w) for w in D.philox4x32(counter, key)) == words


def test_bits_depend_on_their_own_place_alone():
    wide = D.bits(9, 100, 77, 3, 4)
    assert np.array_equal(D.bits(5, 41, 77, 3, 4), wide[:5, :41])
    for other in (D.bits(9, 100, 78, 3, 4), D.bits(9, 100, 77 + (1 << 40), 3, 4), D.bits(9, 100, 77, 2, 4),
                  D.bits(9, 100, 77, 3, 5)):
        assert (other == wide).mean() < 0.02


def test_mask_is_binomial():
    b = D.bits(500, 800, 12345)
    n = b.size
    for p in (0.1, 0.5, 0.9):
        t = D.limit(p)
        share, q = float((b < t).mean()), t / 65536
        assert abs(share - q) < 5 * np.sqrt(q * (1 - q) / n)
    # all 256 values of each byte equally likely: chi-square with 255 degrees of freedom, five deviations
    for byte in (b & 255, b >> 8):
        chi = float((((np.bincount(byte.ravel(), minlength=256) - n / 256) ** 2) / (n / 256)).sum())
        assert abs(chi - 255) < 5 * np.sqrt(2 * 255)


def test_ends_of_the_probability():
    x = np.arange(1.0, 41.0).reshape(4, 10)
    assert np.array_equal(D.dropout(x, 0.0, 1), x)
    assert np.array_equal(D.dropout(x, 1.0, 1), np.zeros_like(x))
    assert D.limit(0.1) == 6554 and D.limit(1e-6) == 0 and D.limit(1 - 1e-6) == 65536
