"""Pins of the oracle's selection where logits are far from zero: values by decimals of eighty digits."""
from decimal import Decimal, getcontext

import numpy as np
import pytest

from oracle import several

F32 = float(np.finfo(np.float32).max)


def _values(x, score):
    getcontext().prec = 80
    xs = [Decimal(float(v)) for v in x]
    m = max(xs)
    lse = m + sum((v - m).exp() for v in xs).ln()
    return [Decimal(float(score)) + v - lse for v in xs]


@pytest.mark.parametrize("x", [[0.0, -1e30, 1.0, -1e30], [-1e30] * 5, [-F32] * 3, [F32, F32, -1e30], [1e9, 1e9 - 64, -5.0],
                               [-7e8, -7e8 - 64, -7e8], [5e30, -F32, 5e30], [1e30, 1.0, 5.0, 1.0, 3.0]])
def test_values_of_rows_far_from_zero(x):
    x = np.array(x, np.float32).astype(np.float64)
    W = len(x)
    logits = np.full((W, len(x)), np.nan)
    logits[0] = x
    got, good = several.select(logits, [-1.25] + [-np.inf] * (W - 1), [0] * W, -1)
    v = _values(x, -1.25)
    order = sorted(range(W), key=lambda t: (-v[t], t))
    assert good and [g[1] for g in got] == order
    for (_, t, s, _) in got:
        assert abs(Decimal(s) - v[t]) <= abs(v[t]) * Decimal(2.0 ** -50) + Decimal(2.0 ** -50)


def test_a_value_below_fp32_is_no_candidate():
    logits = np.array([[1e33, -F32, -F32], [0.0] * 3, [0.0] * 3])
    got, good = several.select(logits, [0.0, -np.inf, -np.inf], [0] * 3, -1)
    assert good and got == [(0, 0, 0.0, 0), (-1, -1, -np.inf, 0), (-1, -1, -np.inf, 0)]
