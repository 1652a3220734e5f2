"""The reference of the operators on logits against hand-worked rows, brute force and differences."""
import itertools
import math

import numpy as np
import pytest

from oracle import logits_ref as L

INF, NAN = math.inf, math.nan


def test_order_by_hand():
    assert L.order_of([1.0, 3.0, NAN, 3.0, -INF, -0.0, 0.0]).tolist() == [1, 3, 0, 5, 6]
    values, classes, rest = L.top_row([0.0, math.log(2.0), -INF], 3)
    assert classes.tolist() == [1, 0, -1] and values[2] == -INF and rest == 0.0
    assert L.top_row([0.0, math.log(2.0), 0.0], 1)[2] == pytest.approx(0.5, rel=1e-15)


@pytest.mark.parametrize("u,T,k,p,m,want", [
    # probabilities 0.1, 0.4, 0.2, 0.3 in the order of the indexes
    (0.0, 1, 0, 1, 0, 0), (0.0999, 1, 0, 1, 0, 0), (0.11, 1, 0, 1, 0, 1), (0.51, 1, 0, 1, 0, 2), (0.71, 1, 0, 1, 0, 3), (1.0, 1, 0, 1, 0, 3),
    (0.999, 1, 1, 1, 0, 1), (0.5, 1, 2, 1, 0, 1), (0.58, 1, 2, 1, 0, 3),          # 0.4, 0.3
    (0.58, 1, 0, 0.5, 0, 3), (0.4, 1, 0, 0.39, 0, 1), (0.4, 1, 0, 0.0, 0, 1),      # 0.4 alone is not 0.5, but is 0.39
    (0.58, 1, 0, 1, 0.7, 3), (0.9, 1, 0, 1, 0.8, 1), (0.9, 1, 0, 1, 7.0, 1),
    (0.3, 0, 0, 1, 0, 1), (0.3, NAN, 0, 1, 0, 1), (0.26, INF, 0, 1, 0, 1), (NAN, 1, 0, 1, 0, 0)])
def test_sample_by_hand(u, T, k, p, m, want):
    assert L.sample_row(np.log([0.1, 0.4, 0.2, 0.3]), u, T, k, p, m)[0] == want


def test_sample_draws_with_the_probabilities_of_the_candidates():
    z = np.array([0.3, -1.0, 2.0, 1.1, -INF, 0.3])
    for T, k, p in itertools.product((0.5, 1.0, 2.0), (0, 2, 3), (1.0, 0.6)):
        n = 20000
        got = np.bincount([L.sample_row(z, (i + 0.5) / n, T, k, p)[0] for i in range(n)], minlength=6) / n
        w = [math.exp(v / T) if v > -INF else 0.0 for v in z]
        rank = sorted(range(6), key=lambda j: (-z[j], j))
        kept, before = [], 0.0
        for i, j in enumerate(rank):
            if (k == 0 or i < k) and (i == 0 or before < p * sum(w)):
                kept.append(j)
            before += w[j]
        want = np.array([w[j] / sum(w[i] for i in kept) if j in kept else 0.0 for j in range(6)])
        assert np.abs(got - want).max() <= 1.0 / n, (T, k, p)


def _loss_by_hand(z, entries, rest, T):
    q = [math.exp(v / T) for v in z]
    q = [v / sum(q) for v in q]
    p = {c: math.exp(v / T) for c, v in entries}
    p = {c: (1 - rest) * v / sum(p.values()) for c, v in p.items()}
    out = sum(v * math.log(v / q[c]) for c, v in p.items() if v > 0)
    left = sum(v for c, v in enumerate(q) if c not in p)
    return out + (rest * math.log(rest / left) if rest > 0 else 0.0)


@pytest.mark.parametrize("rest", [0.0, 0.2, 0.9])
@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_distill_by_hand_and_by_differences(rest, T):
    z = np.array([0.4, -1.2, 2.0, 0.0, 1.5, -0.3])
    values, classes = [1.0, 0.2, -7.0, 3.0, 9.0], [4, 2, 4, -1, 6]    # one twice, two that do not exist
    loss, grad, size = L.distill_row(z, values, classes, rest, T)
    assert loss == pytest.approx(_loss_by_hand(z, [(4, 1.0), (2, 0.2)], rest, T), rel=1e-13)
    for j in range(6):
        d = np.eye(6)[j] * 1e-5
        diff = (L.distill_row(z + d, values, classes, rest, T)[0] - L.distill_row(z - d, values, classes, rest, T)[0]) / 2e-5
        assert grad[j] == pytest.approx(diff, abs=1e-9)
        assert abs(grad[j]) <= size[j] * (1 + 1e-12)


def test_distill_is_zero_for_the_teacher_itself_and_for_empty_rows():
    z = np.array([0.4, -1.2, 2.0, 0.0])
    values, classes, rest = L.top_row(z, 2)
    loss, grad, _ = L.distill_row(z, values, classes, rest)
    assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
    for row, entries in (([-INF] * 3, [0, 1]), ([1.0, 2.0, 3.0], [-1, 3])):
        loss, grad, _ = L.distill_row(row, [1.0, 2.0], entries, 0.3)
        assert loss == 0.0 and not grad.any()
    assert L.distill_row([1.0, 2.0], [-INF, -INF], [0, 1])[0] == 0.0
    assert L.distill_row([-INF, 2.0, 1.0], [1.0, 2.0], [0, 1])[0] == INF
    assert math.isnan(L.distill_row([NAN, 2.0], [1.0], [1])[0])
