"""The random bits that round the roots of second moments: even, and those of the coarse form where that is due."""
import numpy as np
import pytest

from oracle import router as o


@pytest.mark.parametrize("low", [0, 1, 0x7ff, 0xabc, 0xfff])
def test_the_further_bits_are_even_for_every_value_of_the_first(low):
    """Over all 2^20 words with the same lower 12 bits every value of the 8 bits more occurs equally often."""
    words = np.arange(1 << 20, dtype=np.uint64) << np.uint64(12) | np.uint64(low)
    bits = o.root_bits(words, 0.9999)
    assert (bits >> 8 == low).all() and (np.bincount(bits & 255, minlength=256) == 4096).all()


def test_both_forms():
    words = o.noise(np.arange(1 << 20, dtype=np.uint64), 3)
    for beta2, fine in ((0.9, False), (0.999, False), (1 - 2.0 ** -10, False), (1 - 0.99 * 2.0 ** -10, True), (0.99999, True)):
        bits = o.root_bits(words, beta2)
        assert bits.min() >= 0 and bits.max() < 1 << 20
        assert ((bits & 255 == 128).all()) != fine
        # the mean of n even numbers below 2^20: 6 standard errors
        assert abs(bits.mean() / 2.0 ** 20 - 0.5) < 6 * 0.289 / 2.0 ** 10
