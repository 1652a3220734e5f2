"""Sampling whose cut lies next to logit 0, with a maximum and a temperature for which an interval of the grid ends there to
within 1e-15 (tests/test_host_logit_grid.py has the borders themselves), against the definition in 64 bits."""
import numpy as np
import pytest

import paper_2306_17266_amd as S
from tests.test_gpu_logits import check_sample, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [300, 1000, 5003, 16001, 90001])
@pytest.mark.parametrize("T", [0.369084835, 3.98032665])
def test_cut_next_to_logit_zero(n, T):
    ctx = S.Sushi(0)
    rng = np.random.default_rng(n)
    ks = [1, 2, 60, 100, n // 4, n // 2, n // 2 + 1, n - 3]
    rows = len(ks)
    for i, z in enumerate((rng.uniform(-0.05, 0.05, (rows, n)), rng.standard_normal((rows, n)) * 1e-3, rng.standard_normal((rows, n)) * 1e-20,
                           rng.choice([-1e-3, 0.0, 1e-3], (rows, n)))):
        z[:, n // 3] = 11.7255468
        z = z.astype(np.float32)
        u = rng.random(rows)
        view, temperature = put(z, "fp32"), np.full(rows, T)
        # the filters that can cut there: the count, the mass, and the ratio of logit 0 to the maximum (which a logit misses by 1e-9 and
        # more but in the third and fourth set, where it is moved away from logit 0)
        ratio = np.exp(-11.7255468 / T) * (1.0 if i < 2 else 0.9)
        # (T = 0.37: the maximum has all the mass, and only a share of 1 - 1e-7 or a count cuts)
        for what, more in (("k", dict(top_k=ks)), ("p", dict(top_p=np.linspace(0.5, 0.9999999, rows))), ("min", dict(min_p=np.full(rows, ratio)))):
            print("border", n, T, i, what, flush=True)
            check_sample(ctx, z, view, u, (n, T, i, what), temperature=temperature, **more)
    ctx.close()
