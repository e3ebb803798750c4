"""What rounding to 4 bits costs a product, as the README states it."""
import numpy as np

from tests import lowbit_ref, rows_ref


def test_cost_of_4_bits_on_both_sides_and_on_the_weights():
    """Root mean square of a random product's error over the product's.  128 x 2048 and 256 x 2048 values leave 0.5 % of either
    (an error is the mean of 2.6e5 squares at least, the largest row scales shared by a row of 2048): 2 % are allowed."""
    g = np.random.default_rng(5)
    x, w = g.standard_normal((128, 2048)), 0.02 * g.standard_normal((256, 2048))
    y = x @ w.T
    cost = lambda v: np.sqrt(((v - y) ** 2).mean() / (y ** 2).mean())  # noqa: E731
    x4, w4 = (rows_ref.f4_values(v.astype(np.float32)) for v in (x, w))
    assert abs(cost(x4 @ w4.T) / 0.134 - 1) < 0.02
    assert abs(cost(x @ lowbit_ref.quantize4(w.astype(np.float32), 128).T.astype(np.float64)) / 0.117 - 1) < 0.02
