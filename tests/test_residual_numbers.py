"""The numbers of dropout and of stochastic 4-bit coding in the tests' plain forms are those of the codec's CPU implementation."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle  # noqa: E402
from tests import residual_plain as plain  # noqa: E402


@pytest.mark.parametrize("seed", [0, 1, 0xFEDCBA9876543210, (1 << 64) - 1])
@pytest.mark.parametrize("first", [0, 1, 7, (1 << 32) - 10, (1 << 34) - 1001, 5 * (1 << 34) - 3, (1 << 63) - 500, (1 << 64) - 777])
def test_draws_are_the_upper_bits_of_the_codecs_words(seed, first):
    rows, cols = 13, 157
    want = oracle.rng_words(seed, first, rows * cols) >> 8
    assert np.array_equal(plain.draws(rows, cols, seed, first, "cpu").numpy(), want.reshape(rows, cols))
