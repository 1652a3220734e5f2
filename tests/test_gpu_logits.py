"""The operators on logits (sushi_sample, sushi_top_logits, sushi_distill) against their definitions in 64 bits
(oracle/logits_ref.py).  Classes have to be the same everywhere; what the computed numbers may be off by stands at each."""
import math

import numpy as np
import pytest
import torch

import paper_2306_17266_amd as S
from oracle import logits_ref as L
from tests.logits_cases import CONTENTS, round_to as rows_of_type, rows_of

pytestmark = pytest.mark.gpu

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
# Below 2^-126 the steps are equal, 2^-126 times a step at 1 (2^-23, 2^-7): a value there is rounded by up to half of one.
HALF_STEP_SMALL = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134}
# one element, around pieces of 16 bytes, around a workgroup's width, classes of the SuperNets, one and several parts of a row
SIZES = [1, 2, 3, 7, 8, 9, 10, 63, 257, 1000, 1023, 2049, 8193, 16385, 33333, 70001, 140003]


@pytest.fixture(scope="module")
def ctx():
    c = S.Sushi(0)
    yield c
    c.close()


def put(z, dtype, stride=None, offset=0):
    """z on the device as rows of that stride that begin `offset` elements behind an allocation's start; what lies between
    the rows is NaN."""
    rows, n = z.shape
    stride = stride or n
    flat = torch.full((offset + rows * stride + 8,), math.nan, dtype=TORCH[dtype], device="cuda")
    view = flat[offset:offset + rows * stride].view(rows, stride)[:, :n]
    view.copy_(torch.from_numpy(np.ascontiguousarray(z)))
    return view


def floats(v):
    return None if v is None else torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).cuda()


def workspace(rows, n):
    """Of the exact size, filled with ones: nothing may depend on what it holds."""
    return torch.full((S.sushi_logits_workspace(rows, n),), 255, dtype=torch.uint8, device="cuda")


def sample(ctx, view, u, **params):
    rows, n = view.shape
    params = {k: (torch.from_numpy(np.asarray(v, dtype=np.int32)).cuda() if k == "top_k" else floats(v)) for k, v in params.items() if v is not None}
    classes = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    logs = torch.full((rows,), math.nan, device="cuda")
    ctx.sushi_sample(view, floats(u), classes, logs, workspace=workspace(rows, n), **params)
    return classes.cpu().numpy(), logs.cpu().numpy()


def check_sample(ctx, z, view, u, what, only=None, **params):
    classes, logs = sample(ctx, view, u, **params)
    for r in only or range(z.shape[0]):
        p = {k: float(np.float32(v[r])) for k, v in params.items() if v is not None}
        want, log = L.sample_row(z[r], float(np.float32(u[r])), T=p.get("temperature", 1.0), top_k=int(p.get("top_k", 0)),
                                 top_p=p["top_p"] if "top_p" in p and p["top_p"] == p["top_p"] else 1.0,
                                 min_p=p["min_p"] if "min_p" in p and p["min_p"] == p["min_p"] else 0.0)
        assert classes[r] == want, (what, r, p, u[r])
        # a sum of n weights, each off by 2^-43 at most, is at least 1; then a rounding to 24 bits
        off = 2.0 ** -24 * abs(log) + z.shape[1] * 2.0 ** -43 if log > -math.inf else 0.0
        assert logs[r] == log or abs(logs[r] - log) <= off, (what, r, logs[r], log)


def filters(rows, seed):
    rng = np.random.default_rng(seed)
    return dict(temperature=rng.choice([0.3, 0.7, 1.0, 2.0], rows), top_k=rng.choice([0, 1, 2, 5, 40, 300], rows),
                top_p=rng.choice([0.1, 0.5, 0.9, 0.99], rows), min_p=rng.choice([0.0, 0.01, 0.2], rows))


SETS = [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("temperature", "top_k", "top_p", "min_p"), ("temperature", "top_p")]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_sample_sizes(ctx, dtype, n):
    rows = 5
    for i, names in enumerate(SETS):
        z = rows_of("peaks", rows, n, dtype, 100 * n + i)
        u = np.random.default_rng(n + i).random(rows)
        view = put(z, dtype, n + i, i)
        print("sample", dtype, n, names, flush=True)
        check_sample(ctx, z, view, u, (n, names), **{k: v for k, v in filters(rows, n + i).items() if k in names})


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", CONTENTS)
@pytest.mark.parametrize("n", [13, 1000, 5003, 90001])
def test_sample_contents(ctx, dtype, kind, n):
    rows = 6
    for i, names in enumerate(SETS):
        z = rows_of(kind, rows, n, dtype, 7 * n + i)
        u = np.random.default_rng(n + i).random(rows)
        print("sample", dtype, kind, n, names, flush=True)
        check_sample(ctx, z, put(z, dtype), u, (kind, n, names), **{k: v for k, v in filters(rows, n + 10 * i).items() if k in names})


@pytest.mark.parametrize("n", [5, 1000, 70001])
def test_sample_parameters_at_their_ends(ctx, n):
    nan, inf = math.nan, math.inf
    z1 = rows_of("peaks", 1, n, "fp32", n)
    for name, values in (("temperature", [0.0, -1.0, nan, inf, 1e-30, 1e-3, 1e30, 1e-45]), ("top_k", [0, -3, 1, n, n + 1, 2 ** 31 - 1, n - 1, 4]),
                         ("top_p", [0.0, -1.0, nan, 1.0, 2.0, 1e-9, 0.9999999, inf]), ("min_p", [0.0, -1.0, nan, 1.0, 2.0, 1e-30, 1e-3, inf])):
        z = np.repeat(z1, len(values), 0)
        for u in (0.37, 0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0):
            print("sample", name, u, flush=True)
            check_sample(ctx, z, put(z, "fp32"), np.full(len(values), u), (name, u), **{name: values})
    classes, _ = sample(ctx, put(z1, "fp32"), [nan])
    assert classes[0] == L.sample_row(z1[0], 0.0)[0]


def test_sample_every_draw_of_a_row(ctx):
    """One row, 4096 random numbers that go evenly through [0, 1): every class as often as it should be."""
    z1 = rows_of("peaks", 1, 1000, "fp32", 3)
    z = np.repeat(z1, 4096, 0)
    u = (np.arange(4096) + 0.5) / 4096
    for params in (dict(), dict(top_k=np.full(4096, 30)), dict(top_p=np.full(4096, 0.8))):
        check_sample(ctx, z, put(z, "fp32"), u, "every draw", **params)


def check_top(ctx, z, view, k, T, what, only=None):
    rows, n = z.shape
    values = torch.full((rows, k), math.nan, device="cuda")
    classes = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    rest = torch.full((rows,), math.nan, device="cuda")
    ctx.sushi_top_logits(view, values, classes, rest, temperature=T, workspace=workspace(rows, n))
    values, classes, rest = values.cpu().numpy(), classes.cpu().numpy(), rest.cpu().numpy()
    for r in only or range(rows):
        want = L.top_row(z[r], k, float(np.float32(T)))
        assert np.array_equal(classes[r], want[1]), (what, r)
        assert np.array_equal(values[r], want[0].astype(np.float32)), (what, r)
        # weights are off by 5e-9 of themselves at most, in numerator and denominator, or by 2^-1022 where they are that small
        assert abs(rest[r] - want[2]) <= (2.0 ** -24 + 1.2e-8) * want[2] + 1e-45, (what, r, rest[r], want[2])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_top_sizes(ctx, dtype, n):
    for i, k in enumerate(sorted({1, 2, 5, 64, 255, 256, 257, 700, 1024, n - 1, n})):
        if 1 <= k <= min(n, 1024):
            z = rows_of("peaks", 3, n, dtype, 10 * n + k)
            print("top", dtype, n, k, flush=True)
            check_top(ctx, z, put(z, dtype, n + i, i), k, 1.0, (n, k))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", CONTENTS)
@pytest.mark.parametrize("n", [13, 1000, 5003, 90001])
def test_top_contents(ctx, dtype, kind, n):
    for k, T in ((1, 1.0), (7, 3.0), (13, 1e-3), (300, 1.0), (1000, 1e10)):
        if k <= n:
            z = rows_of(kind, 4, n, dtype, n + k)
            print("top", dtype, kind, n, k, flush=True)
            check_top(ctx, z, put(z, dtype), k, T, (kind, n, k))


def teacher_of(z, k, seed, T, spoil=False):
    """(values, classes, rest) of a teacher that mostly agrees; spoil: entries twice, out of range, padding, in any order."""
    rng = np.random.default_rng(seed)
    rows, n = z.shape
    t = np.where(np.isfinite(z), np.clip(z, -50, 50), -3.0) + 0.5 * rng.standard_normal(z.shape)
    got = [L.top_row(t[r].astype(np.float32), k, T) for r in range(rows)]
    values, classes, rest = (np.stack([g[i] for g in got]) for i in range(3))
    if spoil:
        for r in range(rows):
            move = rng.permutation(k)
            values[r], classes[r] = values[r][move], classes[r][move]
        if k >= 4:
            classes[:, k // 2] = classes[:, 0]
            classes[:, 1] = rng.choice([-1, n, 2 ** 31 - 1, -2 ** 31], rows)
            values[0, 2] = -np.inf
        classes[-1] = -1
    return values.astype(np.float32), classes.astype(np.int32), rest.astype(np.float32)


def check_distill(ctx, z, dtype, teacher, T, what, weight=None, in_place=False, stride=None, offset=0, forward_only=False, only=None):
    values, classes, rest = teacher
    rows, n = z.shape
    view = put(z, dtype, stride, offset)
    loss = torch.full((rows,), 7.0, device="cuda")
    grad = view if in_place else put(np.full_like(z, 7.0), dtype, stride, offset)
    ctx.sushi_distill(view, torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), loss, rest=floats(rest), temperature=T,
                      weight=floats(weight), grad=None if forward_only else grad, workspace=workspace(rows, n))
    loss, grad = loss.cpu().numpy().astype(np.float64), grad.float().cpu().numpy().astype(np.float64)
    T = float(np.float32(T))
    for r in only or range(rows):
        want, g, size = L.distill_row(z[r], values[r], classes[r], 0.0 if rest is None else float(rest[r]), T)
        # R is off by 5e-9 of itself at most, and with it ln S, and rest * ln R
        ok = loss[r] == want or (math.isnan(loss[r]) and math.isnan(want)) or abs(loss[r] - want) <= 2.0 ** -24 * abs(want) + 2e-8
        assert ok, (what, r, loss[r], want)
        if forward_only:
            continue
        w = 1.0 if weight is None else float(np.float32(weight[r]))
        if w == 0.0:
            assert not grad[r].any(), (what, r)
            continue
        g, size = g * w, size * abs(w)
        # a weight in 32 bits: the exponent x is a product of three rounded factors (|x| 3 half steps, in units of log2), the
        # exponential is off by a step, and two products are rounded; below 2^-126 it may be zero.  Then the type's rounding.
        with np.errstate(invalid="ignore"):
            x = np.minimum(np.abs(np.where(np.isfinite(z[r]), z[r].astype(np.float64) - np.max(z[r]), 0.0)) / T * 1.4427, 150.0)
            off = size * (2.1 * x + 4.0) * 2.0 ** -24 + HALF_STEP[dtype] * np.abs(g) * 1.001 + abs(w) / T * 2.0 ** -125 + HALF_STEP_SMALL[dtype]
            bad = ~((np.abs(grad[r] - g) <= off) | (np.isnan(grad[r]) & np.isnan(g)))
        assert not bad.any(), (what, r, np.flatnonzero(bad)[:5], grad[r][bad][:5], g[bad][:5], off[bad][:5])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_distill_sizes(ctx, dtype, n):
    for i, (k, with_rest, T) in enumerate(((1, False, 1.0), (5, True, 1.0), (20, True, 2.0), (64, False, 4.0), (257, True, 0.7), (1024, True, 2.0))):
        if k <= n:
            z = rows_of("peaks", 3, n, dtype, 10 * n + k)
            values, classes, rest = teacher_of(z, k, n + k, T)
            print("distill", dtype, n, k, flush=True)
            check_distill(ctx, z, dtype, (values, classes, rest if with_rest else None), T, (n, k), stride=n + i, offset=i,
                          weight=None if i % 2 else np.array([1.0, 0.0, -0.25]), in_place=i % 3 == 1, forward_only=i == 4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", CONTENTS)
@pytest.mark.parametrize("n", [13, 1000, 33333])
def test_distill_contents(ctx, dtype, kind, n):
    for k, T in ((1, 1.0), (7, 3.0), (13, 0.5), (300, 1.0)):
        if k <= n:
            z = rows_of(kind, 4, n, dtype, n + k)
            for spoil in (False, True):
                values, classes, rest = teacher_of(z, k, n + k, T, spoil)
                print("distill", dtype, kind, n, k, spoil, flush=True)
                check_distill(ctx, z, dtype, (values, classes, rest), T, (kind, n, k, spoil))
                check_distill(ctx, z, dtype, (values, classes, None), T, (kind, n, k, spoil, "no rest"))


# long rows: held where there are many, in small parts where there are few, in large parts; in one launch and in several
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", [(2, 32003), (200, 15001), (200, 31001), (200, 65001), (70, 70001), (2, 1 << 20), (70, 1 << 20)])
def test_forms_of_long_rows(ctx, dtype, rows, n):
    z2 = rows_of("peaks", 2, n, dtype, n + rows)
    values, classes, rest = teacher_of(z2, 40, n, 1.0)
    turn = np.arange(rows) % 2
    z, values, classes, rest = z2[turn], values[turn], classes[turn], rest[turn]
    only = sorted({0, 1, rows // 2, 62 % rows, 63 % rows, 64 % rows, rows - 1})
    view, u, f = put(z, dtype), np.random.default_rng(n).random(rows), filters(rows, n)
    for names in SETS:
        print("forms", dtype, rows, n, names, flush=True)
        check_sample(ctx, z, view, u, (rows, n, names), only=only, **{k: v for k, v in f.items() if k in names})
    for k in (1, 40, 1024):
        print("forms, top", dtype, rows, n, k, flush=True)
        check_top(ctx, z, view, k, 1.0, (rows, n, k), only=only)
    del view
    for more in (dict(), dict(in_place=True), dict(forward_only=True)):
        print("forms, distill", dtype, rows, n, more, flush=True)
        check_distill(ctx, z, dtype, (values, classes, rest), 1.0, (rows, n, more), only=only, **more)


def test_distill_teachers_at_their_ends(ctx):
    nan, inf = math.nan, math.inf
    z = rows_of("normal", 8, 1000, "fp32", 5)
    values, classes, _ = teacher_of(z, 6, 5, 1.0)
    check_distill(ctx, z, "fp32", (values, classes, np.array([0.0, 1.0, 0.5, 1e-30, 1.0 - 2.0 ** -24, 2.0, -1.0, nan])), 1.0, "rest")
    values[0] = -inf
    values[1, 3] = inf
    values[2, 0] = nan
    values[3, :5] = -inf
    values[4] = 3.0e38
    values[5] = [200.0, -200.0, 0.0, 1.0, 2.0, 3.0]
    check_distill(ctx, z, "fp32", (values, classes, np.full(8, 0.25)), 1.0, "values")
    check_distill(ctx, z, "fp32", (values, classes, None), 2.0, "values, no rest")
    # the list is the whole row
    z = rows_of("normal", 3, 10, "bf16", 6)
    values, classes, rest = teacher_of(z, 10, 6, 1.0)
    assert not rest.any()
    check_distill(ctx, z, "bf16", (values, classes, rest), 1.0, "whole row")
    check_distill(ctx, z, "bf16", (values, classes, np.full(3, 0.5, np.float32)), 1.0, "mass outside a list of all classes")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", [(5, 1000), (5, 33333), (300, 5000)])
def test_distill_students_sure_of_the_list(ctx, dtype, rows, n):
    """The classes that are not listed have next to nothing, the teacher's mass outside its list all the same: weights far below
    2^-126 of the largest are divided by their own sum."""
    rng = np.random.default_rng(n)
    values, classes, _ = teacher_of(rows_of("peaks", 2, n, dtype, n), 8, n, 1.0)
    turn = np.arange(rows) % 2
    values, classes = values[turn], classes[turn]
    for gap, T in ((60, 1.0), (88, 1.0), (110, 1.0), (300, 1.0), (600, 1.0), (30, 0.1), (64, 0.1), (6, 0.01)):
        z = rng.standard_normal((rows, n)).astype(np.float32) * np.float32(T)
        z[np.arange(rows)[:, None], classes] += np.float32(gap)
        z = rows_of_type(z, dtype)
        for rest in (np.float32([0.3, 1e-6, 1.0]), None):
            print("sure", dtype, n, gap, T, flush=True)
            check_distill(ctx, z, dtype, (values, classes, None if rest is None else rest[np.arange(rows) % 3]), T, (n, gap, T),
                          weight=np.float32([1.0, -1e-3, 1e4, 0.0])[np.arange(rows) % 4], only=list(range(min(rows, 12))))


def test_distill_gradient_against_differences_of_the_loss(ctx):
    """Differences of the definition's loss, h = 1e-4: off by h^2 / 6 times the third derivative (at most 1 here: T >= 1), 2e-9,
    plus the loss's own 64-bit rounding through 2 h."""
    z = rows_of("normal", 2, 12, "fp32", 8)
    values, classes, rest = teacher_of(z, 4, 8, 2.0)
    rest = np.maximum(rest, np.float32(0.05))
    view = put(z, "fp32")
    loss, grad = torch.empty(2, device="cuda"), torch.empty(2, 12, device="cuda")
    ctx.sushi_distill(view, torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), loss, rest=floats(rest), temperature=2.0,
                      grad=grad, workspace=workspace(2, 12))
    for r in range(2):
        for j in range(12):
            d = np.eye(12)[j] * 1e-4
            up, down = (L.distill_row(z[r].astype(np.float64) + s * d, values[r], classes[r], float(rest[r]), 2.0)[0] for s in (1, -1))
            assert abs(float(grad[r, j]) - (up - down) / 2e-4) <= 1e-6, (r, j)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_behind_the_last_and_between_rows_stay_as_they_were(ctx, dtype):
    rows, n, stride = 3, 1001, 1024
    z = rows_of("peaks", rows, n, dtype, 9)
    values, classes, _ = teacher_of(z, 8, 9, 1.0)
    view = put(z, dtype, stride, 3)
    flat = torch.full((3 + rows * stride + 64,), 7.0, dtype=TORCH[dtype], device="cuda")
    grad = flat[3:3 + rows * stride].view(rows, stride)[:, :n]
    loss = torch.full((rows + 2,), 7.0, device="cuda")
    ctx.sushi_distill(view, torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), loss[:rows], grad=grad, workspace=workspace(rows, n))
    grad.fill_(7.0)
    assert bool((flat == 7.0).all()) and bool((loss[rows:] == 7.0).all())
    out = torch.full((rows + 2, 9), 7.0, device="cuda")
    index = torch.full((rows + 2, 9), 7, dtype=torch.int32, device="cuda")
    ctx.sushi_top_logits(view, out[:rows], index[:rows], loss[:rows], workspace=workspace(rows, n))
    assert bool((out[rows:] == 7.0).all()) and bool((index[rows:] == 7).all()) and bool((loss[rows:] == 7.0).all())


def test_a_run_of_them_after_queries(ctx):
    """What a program does: queries of the largest and of a smaller SubNet, the teacher's list from one, the loss and gradient
    of the other, an answer for each image."""
    from tests.common import make_problem
    from workloads import arch as A
    from workloads import tensors as T
    arch = A.tiny_arch()
    blob, _ = make_problem(arch, 4, False)
    c = S.Sushi(0)
    c.sushi_load_supernet(arch, blob, S.FP32)
    batch = 6
    x = torch.from_numpy(T.make_input(4, 0, batch, 32, 3, False)).cuda()
    big, small = (torch.empty(batch, arch.n_classes, device="cuda") for _ in range(2))
    values, classes = torch.empty(batch, 4, device="cuda"), torch.empty(batch, 4, dtype=torch.int32, device="cuda")
    rest, loss, grad = torch.empty(batch, device="cuda"), torch.empty(batch, device="cuda"), torch.empty_like(small)
    answer, u = torch.empty(batch, dtype=torch.int32, device="cuda"), torch.rand(batch, device="cuda")
    work = workspace(batch, arch.n_classes)
    c.sushi_infer(A.max_cfg(arch, 32), x, big)
    c.sushi_infer(A.min_cfg(arch, 32), x, small)
    c.sushi_top_logits(big, values, classes, rest, temperature=2.0, workspace=work)
    c.sushi_distill(small, values, classes, loss, rest=rest, temperature=2.0, grad=grad, workspace=work)
    c.sushi_sample(small, u, answer, workspace=work)
    c.sushi_synchronize()
    for r in range(batch):
        v, k, q = L.top_row(big[r].cpu().numpy(), 4, 2.0)
        assert classes[r].cpu().tolist() == k.tolist()
        want, g, _ = L.distill_row(small[r].cpu().numpy(), v, k, q, 2.0)
        # (the list's values and mass were rounded to 32 bits on the way, as the test of each operator allows)
        assert abs(float(loss[r]) - want) <= 1e-6 * (1 + abs(want)) and np.abs(grad[r].cpu().numpy() - g).max() <= 1e-6
        assert int(answer[r]) == L.sample_row(small[r].cpu().numpy(), float(u[r]))[0]
    c.close()


@pytest.mark.parametrize("mode,dtype", [(0, "fp32"), (1, "fp32"), (0, "bf16"), (3, "bf16")])
def test_measure_agreement(mode, dtype):
    """Against the definitions, on the logits of the same queries: losses off as in check_distill, after a list rounded to 32 bits."""
    from paper_2306_17266_amd import sushiabs
    from tests.common import make_problem
    from workloads import arch as A
    from workloads import tensors as T
    arch = A.tiny_arch()
    blob, _ = make_problem(arch, 4, dtype == "bf16")
    stream = torch.cuda.Stream()
    c = S.Sushi(0, stream.cuda_stream)
    c.sushi_load_supernet(arch, blob, S.BF16 if dtype == "bf16" else S.FP32)
    c.sushi_set_option(S.OPT_EXEC_MODE, mode)
    xs = [torch.from_numpy(T.make_input(4, i, b, 32, 3, dtype == "bf16")).cuda().to(TORCH[dtype]) for i, b in enumerate((6, 1, 9))]
    subnets = [A.min_cfg(arch, 32), A.max_cfg(arch, 32)]
    torch.cuda.synchronize()
    z = []
    for cfg in subnets:
        out = torch.empty(16, arch.n_classes, device="cuda")
        torch.cuda.synchronize()
        for x, at in zip(xs, (0, 6, 7)):
            c.sushi_infer(cfg, x, out[at:at + len(x)])
        c.sushi_synchronize()
        z.append(out.cpu().numpy())
    u = np.random.default_rng(5).random(16, dtype=np.float32)
    for k, sampling in ((4, None), (64, dict(temperature=3.0, top_k=5, top_p=0.9, min_p=0.01))):
        divergence, agreement = sushiabs.measure_agreement(c, subnets, subnets[1], xs, arch.n_classes, k, 2.0, sampling, seed=5)
        s = dict(T=0.0) if sampling is None else dict(T=3.0, top_k=5, top_p=float(np.float32(0.9)), min_p=float(np.float32(0.01)))
        answers = [[L.sample_row(row, float(u[r]), **s)[0] for r, row in enumerate(rows)] for rows in z]
        for i, rows in enumerate(z):
            losses = [L.distill_row(row, *L.top_row(z[1][r], min(k, arch.n_classes), 2.0), 2.0)[0] for r, row in enumerate(rows)]
            assert abs(divergence[i] - np.mean(losses)) <= 1e-6 * (1 + np.mean(losses))
            assert agreement[i] == np.float32(np.mean(np.equal(answers[i], answers[1])))
        assert divergence[0] > 0.01 and divergence[1] < 1e-6 and agreement[1] == 1.0
    c.close()


@pytest.mark.parametrize("T", [1e-45, 1e-38, 1e-30, 1e30, 3e38])
def test_temperatures_at_their_ends(ctx, T):
    z = rows_of("peaks", 4, 1000, "fp32", 50)
    z[1], z[2] = z[1, 0], -z[2]
    check_top(ctx, z, put(z, "fp32"), 20, T, T)
    values, classes, rest = teacher_of(z, 20, 50, 1.0)
    for r in (rest, None):
        check_distill(ctx, z, "fp32", (values, classes, r), T, T, forward_only=T < 1e-38)  # (1 / T is not a float32 number there)
        check_distill(ctx, z, "fp32", (values, classes, r), T, T, weight=np.float32([1e4, 1, 0, -1e-3]), forward_only=T < 1e-30)


def _all_three(c, z, u, values, classes, out, work):
    c.sushi_sample(z, u, out["class"], out["log"], top_k=out["k"], top_p=out["p"], workspace=work)
    c.sushi_top_logits(z, out["values"], out["classes"], out["rest"], workspace=work)
    c.sushi_distill(z, values, classes, out["loss"], rest=out["rest"], grad=out["grad"], workspace=work)


def _problem(rows, n, dtype, seed):
    z = rows_of("peaks", rows, n, dtype, seed)
    values, classes, _ = teacher_of(z, 9, seed, 1.0)
    out = dict(k=torch.full((rows,), 20, dtype=torch.int32, device="cuda"), p=torch.full((rows,), 0.9, device="cuda"))
    for name, shape, t in (("class", (rows,), torch.int32), ("log", (rows,), torch.float32), ("values", (rows, 9), torch.float32),
                           ("classes", (rows, 9), torch.int32), ("rest", (rows,), torch.float32), ("loss", (rows,), torch.float32),
                           ("grad", (rows, n), TORCH[dtype])):
        out[name] = torch.zeros(shape, dtype=t, device="cuda")
    return put(z, dtype), torch.rand(rows, device="cuda"), torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), out


@pytest.mark.parametrize("rows,n", [(3, 1000), (2, 100003), (300, 5000)])
def test_captured_and_replayed(rows, n):
    """All three in one graph, replayed on new inputs between eager work, against eager calls; twice on the same inputs: bit for bit."""
    stream = torch.cuda.Stream()
    c = S.Sushi(0, stream.cuda_stream)
    z, u, values, classes, out = _problem(rows, n, "fp32", 11)
    work = workspace(rows, n)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        _all_three(c, z, u, values, classes, out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        _all_three(c, z, u, values, classes, out, work)
    for i in range(4):
        z.copy_(torch.from_numpy(rows_of("peaks", rows, n, "fp32", 20 + i)))
        u.copy_(torch.rand(rows, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        work.fill_(i)
        for name in ("class", "log", "values", "classes", "rest", "loss", "grad"):
            out[name].fill_(-3)
        torch.cuda.synchronize()
        _all_three(c, z, u, values, classes, out, work)
        torch.cuda.synchronize()
        for name in out:
            assert torch.equal(got[name], out[name]), (i, name)
    c.close()


def test_two_graphs_share_a_workspace():
    """Replayed in turn on one stream, with eager calls in the same workspace between them: as each by itself."""
    stream = torch.cuda.Stream()
    c = S.Sushi(0, stream.cuda_stream)
    problems = [_problem(3, 90001, "fp32", 60), _problem(40, 1000, "bf16", 61)]
    work = torch.full((max(S.sushi_logits_workspace(3, 90001), S.sushi_logits_workspace(40, 1000)),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    want, graphs = [], []
    for p in problems:
        _all_three(c, *p, work)
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in p[-1].items()})
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            _all_three(c, *p, work)
    for i in range(4):
        for p in problems:
            for name in ("class", "log", "values", "classes", "rest", "loss", "grad"):
                p[-1][name].fill_(-3)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graphs[i % 2].replay()
            _all_three(c, *problems[i % 2], work)
            graphs[1 - i % 2].replay()
        torch.cuda.synchronize()
        for p, w in zip(problems, want):
            for name in w:
                assert torch.equal(w[name], p[-1][name]), (i, name)
    c.close()


def test_two_streams_at_once():
    """Two contexts with streams and workspaces of their own, their work interleaved: as each by itself."""
    sides = []
    for i in range(2):
        stream = torch.cuda.Stream()
        sides.append((S.Sushi(0, stream.cuda_stream), _problem(2, 90001, "bf16", 30 + i), workspace(2, 90001)))
    torch.cuda.synchronize()
    want = []
    for c, p, work in sides:
        _all_three(c, *p, work)
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in p[-1].items()})
    for _ in range(10):
        for c, p, work in sides:
            _all_three(c, *p, work)
    torch.cuda.synchronize()
    for (c, p, _), w in zip(sides, want):
        for name in w:
            assert torch.equal(w[name], p[-1][name]), name
        c.close()


def test_long_rows_beyond_32_bits(ctx):
    """The last of a few rows that lie 1.1e9 elements apart (bytes and elements pass 2^31 and 2^32)."""
    n, stride, rows = 5003, 1_100_000_000, 3
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GiB of device memory")
    flat = torch.empty(2 * (rows - 1) * stride + 2 * n, dtype=torch.bfloat16, device="cuda")
    z = rows_of("peaks", rows, n, "bf16", 40)
    views = [torch.as_strided(flat, (rows, n), (stride, 1), o) for o in (0, (rows - 1) * stride + n)]
    for v in views:
        v.copy_(torch.from_numpy(z))
    u = np.random.default_rng(1).random(rows)
    check_sample(ctx, z, views[1], u, "far rows", top_p=np.full(rows, 0.9))
    check_top(ctx, z, views[1], 20, 1.0, "far rows")
    values, classes, rest = teacher_of(z, 9, 41, 1.0)
    loss = torch.empty(rows, device="cuda")
    ctx.sushi_distill(views[1], torch.from_numpy(values).cuda(), torch.from_numpy(classes).cuda(), loss, rest=floats(rest),
                      grad=views[0], workspace=workspace(rows, n))
    for r in range(rows):
        want, g, size = L.distill_row(z[r], values[r], classes[r], float(rest[r]))
        assert abs(float(loss[r]) - want) <= 2.0 ** -24 * abs(want) + 2e-8
        assert (np.abs(views[0][r].float().cpu().numpy() - g) <= 2.0 ** -8 * np.abs(g) * 1.01 + size * 1e-5 + 1e-37).all()
