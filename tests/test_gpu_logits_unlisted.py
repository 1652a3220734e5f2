"""sushi_distill where the student gives the classes outside the list next to nothing: their sum is 2^-1000 of the row's and far
less, and loss and gradient are finite all the same.  Against the definition in 64 bits (oracle/logits_ref.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2306_17266_amd as S
from oracle import logits_ref as L
from tests.logits_cases import LOWEST, round_to
from tests.test_gpu_logits import HALF_STEP, HALF_STEP_SMALL, floats, put, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = S.Sushi(0)
    yield c
    c.close()


def check(ctx, z, dtype, values, classes, rest, T, weight, what, in_place=False, rows=None, view=None, grad=None):
    view = put(z, dtype) if view is None else view
    loss, grad = torch.full((z.shape[0],), 7.0, device="cuda"), view if in_place else torch.full_like(view, 7.0) if grad is None else grad
    ctx.sushi_distill(view, torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), loss, rest=floats(rest), temperature=T,
                      weight=floats(weight), grad=grad, workspace=workspace(*z.shape))
    loss, grad = loss.cpu().numpy().astype(np.float64), grad.float().cpu().numpy().astype(np.float64)
    T = float(np.float32(T))
    for r in range(z.shape[0]) if rows is None else rows:
        want, g, size = L.distill_row(z[r], values[r], classes[r], 0.0 if rest is None else float(rest[r]), T)
        # the sums are off by 2e-9 of themselves, which is added to the logarithms; then a rounding to 24 bits
        assert loss[r] == want or abs(loss[r] - want) <= 2.0 ** -24 * abs(want) + 2e-8, (what, r, loss[r], want)
        w = 1.0 if weight is None else float(np.float32(weight[r]))
        others = np.ones(z.shape[1], dtype=bool)
        others[classes[r][(classes[r] >= 0) & (classes[r] < z.shape[1])]] = False
        # An unlisted class: its exponent x, counted from the largest unlisted logit, is the product of two rounded factors, rounded (3
        # half steps of x, ln 2 of it in the weight); the exponential is off by two half steps, the factor and the product by one
        # each, the sums in the factor by 2e-9 each (0.1 half steps).  A weight below 2^-126 may be zero; a factor that small is rounded by
        # up to half of 2^-149.  A listed class has 64 bits.  Then the type's rounding.
        with np.errstate(invalid="ignore"):
            x = np.where(others, np.abs(z[r].astype(np.float64) - z[r][others].max(initial=-np.inf)), 0.0) / T * 1.4426950408889634
            x = np.where(np.isfinite(x), np.minimum(x, 150.0), 150.0)
            off = abs(w) * size * np.where(others, 2.1 * x + 4.1, 0.1) * 2.0 ** -24 + HALF_STEP[dtype] * np.abs(g * w) * 1.001
            off += abs(w) / T * 2.0 ** -125 + 2.0 ** -149 + HALF_STEP_SMALL[dtype]
            bad = ~(np.abs(grad[r] - g * w) <= off)
        assert not bad.any(), (what, r, np.flatnonzero(bad)[:5], grad[r][bad][:5], (g * w)[bad][:5], off[bad][:5])


def student(rng, rows, n, k, gap, T, dtype):
    """Rows whose k listed classes stand gap * T above the others, and the list."""
    classes = np.stack([rng.permutation(n)[:k] for _ in range(rows)]).astype(np.int32)
    z = rng.standard_normal((rows, n)) * 2.0 * T
    z[np.arange(rows)[:, None], classes] += gap * T
    return round_to(z, dtype), (rng.standard_normal((rows, k)) * T).astype(np.float32), classes


FORMS = [(5, 10), (6, 1000), (300, 5000), (4, 9001), (5, 33333), (2, 140003), (70, 70001)]  # held, in small parts, in large parts


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", FORMS)
def test_unlisted_far_below(ctx, dtype, rows, n):
    rng = np.random.default_rng(n)
    some = sorted({0, 1, rows // 2, rows - 1})
    for i, (gap, T) in enumerate(((690, 1.0), (712, 1.0), (750, 0.05), (1000, 1.0), (1000, 0.01), (1e5, 1.0), (1e5, 1e-3), (1e5, 30.0))):
        z, values, classes = student(rng, rows, n, min(8, n // 2), gap, T, dtype)
        rest = np.float32([0.3, 1e-6, 1.0, 0.0])[(np.arange(rows) + i) % 4]
        weight = None if i % 2 else np.float32([1.0, -1e-3, 1e4])[np.arange(rows) % 3]
        print("unlisted", dtype, rows, n, gap, T, flush=True)
        check(ctx, z, dtype, values, classes, rest, T, weight, (rows, n, gap, T), in_place=i % 3 == 2, rows=some)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", FORMS)
def test_masks_of_finite_values(ctx, dtype, rows, n):
    """Everything but the list masked with -1e4 or the type's lowest value: the masked classes share the mass outside the list."""
    rng = np.random.default_rng(n + 1)
    some = sorted({0, 1, rows // 2, rows - 1})
    for mask, T in ((-1e4, 1.0), (LOWEST[dtype], 4.0), (LOWEST[dtype], 1e5)):
        z, values, classes = student(rng, rows, n, min(8, n // 2), 0, 1.0, dtype)
        keep = np.zeros((rows, n), dtype=bool)
        keep[np.arange(rows)[:, None], classes] = True
        z = round_to(np.where(keep, z, mask), dtype)
        z[0, np.flatnonzero(~keep[0])[0]] = -np.inf  # (one of a row is not there at all)
        print("masks", dtype, rows, n, mask, T, flush=True)
        check(ctx, z, dtype, values, classes, np.full(rows, 0.25, np.float32), T, None, (rows, n, mask, T), rows=some)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_levels_between_parts(ctx, dtype):
    """Unlisted logits on levels far apart, a stretch of the row each: parts whose own sums are 2^-1000 of the next one's, parts without
    an unlisted logit above -inf, the largest in the first, a middle and the last part."""
    rng = np.random.default_rng(7)
    n, rows, k = 70001, 6, 5
    z = rng.standard_normal((rows, n)) - 5000.0
    for r, (at, level) in enumerate(((0, -2500.0), (30000, -2500.0), (n - 1, -2500.0), (20000, 900.0), (0, -4999.0), (n - 9, -np.inf))):
        z[r, at:at + 3000] += level + 5000.0 - 2500.0
        z[r, 40000:50000] = -np.inf
    classes = np.stack([rng.permutation(n)[:k] for _ in range(rows)]).astype(np.int32)
    classes[:, 0] = [45000, 100, n - 1, 20001, 0, 3]
    z[np.arange(rows)[:, None], classes] = rng.standard_normal((rows, k))
    z, values = round_to(z, dtype), rng.standard_normal((rows, k)).astype(np.float32)
    for T in (1.0, 0.3):
        for rest in (np.full(rows, 0.2, np.float32), None):
            print("levels", dtype, T, flush=True)
            check(ctx, z, dtype, values, classes, rest, T, None, (T, rest is None))


def test_infinite_logits_beside_the_list(ctx):
    """+inf in the list, outside it, in both: who shares the row, and whether something is left outside."""
    inf = math.inf
    for n in (10, 1000, 40003):
        z = np.random.default_rng(n).standard_normal((4, n)).astype(np.float32)
        z[0, 1], z[1, n - 1], z[2, [1, n - 1]] = inf, inf, inf
        classes = np.tile(np.int32([1, 4]), (4, 1))
        values = np.tile(np.float32([0.5, -0.5]), (4, 1))
        for rest in (np.full(4, 0.2, np.float32), None):
            print("infinite", n, flush=True)
            check(ctx, z, "fp32", values, classes, rest, 1.0, None, (n, rest is None))
