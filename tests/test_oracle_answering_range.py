"""The top of the 4-bit format's range by hand (CPU): nothing finite becomes an infinity."""
import numpy as np

from oracle import answering as A


def test_the_largest_power():
    for x, power, value in ((1.7 * 2.0 ** 127, 252, 6 * 2.0 ** 125), (1.75 * 2.0 ** 127, 252, 6 * 2.0 ** 125),
                            (255 * 2.0 ** 120, 252, 6 * 2.0 ** 125), (2.0 ** 127, 252, 4 * 2.0 ** 125),
                            (0.874 * 2.0 ** 127, 251, 6 * 2.0 ** 124), (0.875 * 2.0 ** 127, 252, 4 * 2.0 ** 125)):
        row = np.zeros(32)
        row[4], row[9] = -x, 2.0 ** 124
        c, e = A.fp4_encode(row)
        held = A.fp4_decode(c, e)
        assert e.tolist() == [power] and held[4] == -value and held[9] == 2.0 ** 124, x
        assert np.all(np.abs(held) < 2.0 ** 128)
