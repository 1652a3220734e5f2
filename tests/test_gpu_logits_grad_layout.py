"""sushi_distill with gradients whose rows lie otherwise than those of the logits: another alignment within 16 bytes, another row
stride.  Against the definition in 64 bits, and what lies around the gradient's rows stays as it was."""
import numpy as np
import pytest
import torch

import paper_2306_17266_amd as S
from tests.logits_cases import rows_of
from tests.test_gpu_logits import SIZES, TORCH, put, teacher_of
from tests.test_gpu_logits_unlisted import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = S.Sushi(0)
    yield c
    c.close()


def check_layout(ctx, dtype, rows, n, z_layout, grad_layout, seed):
    """layout: (elements before the first row, elements between rows)."""
    distinct = min(rows, 4)
    turn = np.arange(rows) % distinct
    z = rows_of("peaks", distinct, n, dtype, seed)
    k = min(n, 20)
    values, classes, rest = teacher_of(z, k, seed, 1.0)
    rest = np.maximum(rest, np.float32(0.01))
    if k == n:
        rest = np.zeros_like(rest)
    z, values, classes, rest = z[turn], values[turn], classes[turn], rest[turn]
    view = put(z, dtype, n + z_layout[1], z_layout[0])
    at, stride = grad_layout[0], n + grad_layout[1]
    flat = torch.full((at + rows * stride + 16,), 7.0, dtype=TORCH[dtype], device="cuda")
    grad = torch.as_strided(flat, (rows, n), (stride, 1), at)
    some = sorted({0, 1 % rows, rows // 2, rows - 1})
    print("layout", dtype, rows, n, z_layout, grad_layout, flush=True)
    check(ctx, z, dtype, values, classes, rest, 1.0, None, (dtype, rows, n, z_layout, grad_layout), rows=some, view=view, grad=grad)
    # (equal rows of a launch have equal gradients: every row was written)
    assert torch.equal(grad, grad[torch.from_numpy(turn).cuda()])
    grad.fill_(7.0)
    assert bool((flat == 7.0).all())


LAYOUTS = [((0, 0), (1, 0)), ((1, 0), (0, 0)), ((0, 0), (0, 1)), ((3, 5), (2, 0)), ((0, 0), (8, 0)), ((0, 3), (0, 11))]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_sizes(ctx, dtype, n):
    for i, (z_layout, grad_layout) in enumerate(LAYOUTS):
        for rows in (1, 3):
            check_layout(ctx, dtype, rows, n, z_layout, grad_layout, n + i)


# in small parts, in one large part a row, in several; in one launch and in more than one
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", [(300, 1000), (1030, 1000), (1030, 9001), (70, 70001), (9000, 37)])
def test_many_rows(ctx, dtype, rows, n):
    for i, (z_layout, grad_layout) in enumerate(LAYOUTS[:4]):
        check_layout(ctx, dtype, rows, n, z_layout, grad_layout, n + i)
