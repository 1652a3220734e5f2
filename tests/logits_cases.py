"""Rows of logits for the tests of the operators on them: sizes and contents where these can go wrong."""
import numpy as np

LOWEST = {"fp32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}


def round_to(x, dtype):
    """float32 values that the type holds (bf16: rounded to nearest even)."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    if dtype == "fp32":
        return x
    u = x.view(np.uint32)
    up = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return np.where(np.isnan(x), x, up.astype(np.uint32).view(np.float32))


def rows_of(kind, rows, n, dtype, seed):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((rows, n)) * rng.uniform(0.5, 4.0, (rows, 1))
    if kind == "peaks":
        z[np.arange(rows)[:, None], rng.integers(0, n, (rows, 8))] += rng.uniform(4, 10, (rows, 8))
    elif kind == "flat":                       # all logits equal
        z[:] = rng.standard_normal((rows, 1))
    elif kind == "few_values":                 # long ties
        z = rng.choice([-1.5, 0.25, 0.75], (rows, n))
    elif kind == "narrow":                     # many different values within a small part of a factor of two
        z = 5.0 + rng.random((rows, n)) * 1e-3
    elif kind == "zeros":                      # of both signs
        z = np.where(rng.random((rows, n)) < 0.5, 0.0, -0.0)
    elif kind == "wide":                       # from one end of the type to the other
        z = rng.standard_normal((rows, n)) * 10.0 ** rng.uniform(-38, 37, (rows, n))
    elif kind == "masked":                     # a third is not there; the first row is empty, the second has one logit
        z[rng.random((rows, n)) < 0.33] = -np.inf
        z[0] = -np.inf
        if rows > 1:
            z[1] = -np.inf
            z[1, n // 2] = 1.0
    elif kind == "lowest":                     # masked with the type's lowest value
        z[rng.random((rows, n)) < 0.33] = LOWEST[dtype]
        z[0] = LOWEST[dtype]
    elif kind == "nan":
        z[rng.random((rows, n)) < 0.1] = np.nan
        z[0] = np.nan
    elif kind == "inf":
        z[:, n // 3] = np.inf
        if rows > 1:
            z[1, n - 1] = np.inf
        z[rng.random((rows, n)) < 0.1] = -np.inf
    else:
        assert kind in ("normal", "peaks"), kind
    return round_to(z, dtype)


CONTENTS = ["normal", "peaks", "flat", "few_values", "narrow", "zeros", "wide", "masked", "lowest", "nan", "inf"]
