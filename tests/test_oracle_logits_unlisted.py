"""The oracle's distillation where the unlisted classes have next to nothing of the student, against 60-digit arithmetic."""
import math
from decimal import Decimal, localcontext

import numpy as np
import pytest

from oracle import logits_ref as L


def by_hand(z, entries, rest, T):
    """loss and gradient from the formulas, in decimal, every probability by its logarithm."""
    with localcontext() as c:
        c.prec, c.Emin, c.Emax = 60, -10 ** 17, 10 ** 17

        def log_sum(x):
            x = list(x)
            return max(x) + sum((v - max(x)).exp() for v in x).ln()

        T, rest = Decimal(T), Decimal(rest)
        z, t = [Decimal(float(v)) / T for v in z], {j: Decimal(float(v)) / T for j, v in entries}
        total, total_t = log_sum(z), log_sum(t.values())
        log_q = [v - total for v in z]
        p = {j: (1 - rest) * (v - total_t).exp() for j, v in t.items()}
        log_q_rest = log_sum(v for j, v in enumerate(log_q) if j not in p)
        loss = sum(v * (v.ln() - log_q[j]) for j, v in p.items() if v > 0)
        if rest > 0:
            loss += rest * (rest.ln() - log_q_rest)
        grad = [(v.exp() - p[j]) / T if j in p else (v.exp() - rest * (v - log_q_rest).exp()) / T for j, v in enumerate(log_q)]
        return float(loss), [float(g) for g in grad]


@pytest.mark.parametrize("T", [1.0, 0.06, 0.055, 0.05, 0.04, 0.01, 0.0004, 1e-30])
@pytest.mark.parametrize("rest", [0.0, 1e-6, 0.3, 1.0])
def test_unlisted_far_below_the_largest(T, rest):
    T, rest = float(np.float32(T)), float(np.float32(rest))
    z, entries = [0.0, -1.0, -40.0, -41.0, -42.5], [(0, 0.5), (1, 0.25)]
    loss, grad, size = L.distill_row(z, [v for _, v in entries], [j for j, _ in entries], rest, T)
    want, g = by_hand(z, entries, rest, T)
    assert loss == pytest.approx(want, rel=1e-13, abs=1e-13)
    assert np.all(np.abs(grad - g) <= 1e-13 * size + 1e-300)


def test_the_example_with_its_figures():
    loss, grad, _ = L.distill_row([0.0, -1.0, -40.0, -41.0, -42.5], [0.0, -1.0], [0, 1], 0.3, 0.05)
    assert loss == pytest.approx(239.3891357, abs=1e-6) and grad[2] == pytest.approx(-6.0, abs=1e-7)


def test_one_step_of_the_range():
    """Losses around the largest float32: finite in its range, infinite beyond."""
    far = np.float32(3.4e38)
    assert L.distill_row([0.0, -far], [0.0], [0], 1.0, 1.0)[0] == pytest.approx(float(far))
    assert L.distill_row([0.0, -far], [0.0], [0], 1.0, 0.5)[0] == math.inf
    assert L.distill_row([0.0, -math.inf], [0.0], [0], 0.5, 1.0)[0] == math.inf
