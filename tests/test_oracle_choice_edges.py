"""Pins of the row-wise choices' oracle far below a row's best score."""
import numpy as np

from oracle import choice_oracle as C


def test_softmax_routing_keeps_the_order_far_below_the_best():
    x = np.array([[0, -40, -30, -50], [-85, 0, -84, -86]], np.float32)
    e, w = C.route(x, 3, "softmax", renorm=False)
    assert e.tolist() == [[0, 2, 1], [1, 2, 0]]
    # |t| <= 126 moved by 2.5 2^-24 |t| ln 2, and under 1e-6 more
    np.testing.assert_allclose(w, np.exp(np.take_along_axis(x, e, 1).astype(np.float64)), rtol=1.5e-5)
    e, w = C.route(x, 2, "softmax", bias=[-2, -2, 0, 0])  # a bias chooses experts of tiny scores
    assert e.tolist() == [[2, 3], [2, 3]]
    np.testing.assert_allclose(w[:, 1], 1 / (1 + np.exp([20.0, 2.0])), rtol=3e-5)
