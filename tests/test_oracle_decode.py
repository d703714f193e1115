"""The draw's oracle against values worked out by hand where logits are infinite."""

import math

import numpy as np

from oracle import decode as oracle


def test_the_oracle_counts_infinity_as_the_largest_number():
    most = float(np.finfo(np.float32).max)
    l = np.array([1.0, most, np.inf, -np.inf, np.nan, most / 2], np.float32)
    assert [oracle.draw(l, u)[0] for u in (0.0, 0.49, 0.5, 0.99)] == [1, 1, 2, 2]
    assert oracle.draw(l, 0.99, temperature=0.0)[0] == 1 and oracle.draw(l, 0.99, top_k=1)[0] == 1
    assert [oracle.draw(l, u, temperature=math.inf)[0] for u in (0.1, 0.3, 0.6, 0.8)] == [0, 1, 2, 5]
    np.testing.assert_allclose(oracle.draw(l, 0.1, temperature=most)[1], math.log(math.exp(-1) / (2 + math.exp(-1) + math.exp(-0.5))))
