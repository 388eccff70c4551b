"""The arithmetic of a raised reference in the 8-bit cache's attention over many
rows, restated: after a raise a chunk's 32 weights fit f16 at any score."""
import numpy as np
import pytest

F = np.float32
UP, MOST, FAR = F(7), 46340.0, F(2.0 ** 22)


def weights(s, f, m):
    """The weights of scores s f relative to m, base 2."""
    if abs(m) >= FAR:
        x = (s * f - m) + UP
    else:                                            # one rounding: exact product and sum in 64 bits and more
        x = (s.astype(np.longdouble) * np.longdouble(f) - np.longdouble(m - UP)).astype(F)
    return np.exp2(x.astype(np.float64))


@pytest.mark.parametrize("exponent", [0, 4, 10, 18, 20, 21, 22, 23, 24, 26, 27, 28, 30, 33, 36, 40, 60, 100])
def test_a_raised_chunk_fits(exponent):
    rng = np.random.default_rng(exponent)
    for _ in range(500):
        s = (rng.standard_normal(32) * 2.0 ** (exponent - 3)).astype(F)
        f = F(rng.uniform(8, 16))
        old = F(np.ceil(rng.standard_normal() * 2.0 ** exponent))
        m = np.maximum(old, np.ceil((s * f).max()))  # as a raise leaves it, or one of long ago
        w = weights(s, f, m)
        assert w.sum() <= 32 * 2.0 ** 7.5 < MOST
        if m > old and abs(m) >= FAR:
            assert 2.0 ** 6 < w.max() <= 2.0 ** 7    # the largest score's, within a whole number, however far
