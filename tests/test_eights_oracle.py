"""CPU-only pins of the oracle's sums of eight neighbouring 8-bit products."""
import numpy as np

from oracle import block_oracle as blk


def test_what_is_cut_off():
    one = np.ones((1, 1))
    x, w = np.zeros((1, 32)), np.zeros((1, 32))
    x[0, :2], w[0, :2] = (256, -256), 256                       # 2^16 - 2^16
    for small, at, kept in ((8.0, 2, 8.0), (4.0, 2, 0.0), (12.0, 7, 8.0), (-12.0, 7, -8.0), (2.0 ** -9, 8, 2.0 ** -9)):
        x2, w2 = x.copy(), w.copy()
        x2[0, at], w2[0, at] = small, 1
        assert blk.eights(x2, one, w2, one)[0][0, 0] == kept


def test_values_of_few_bits_are_added_exactly():
    rng = np.random.default_rng(1)
    x, w = rng.integers(-8, 9, (5, 96)).astype(float), rng.integers(-2, 3, (7, 96)).astype(float)
    xs, ws = np.exp2(rng.integers(-5, 5, (5, 3))), np.exp2(rng.integers(-5, 5, (7, 3)))
    got, size = blk.eights(x, xs, w, ws)
    X, W = blk.mx8_value(x, xs), blk.mx8_value(w, ws)
    assert np.array_equal(got, X @ W.T) and np.array_equal(size, abs(X) @ abs(W).T)
