"""Rows and tolerances shared by the tests of the records of top logits.

Tolerances.  The kernels form 2^((x - top) c2) with v_exp_f32 (1 unit in the
last place) from an exponent whose rounding is at most 2^-24 of it for c2 and
for the product, so a term 2^-n of the largest is off by at most
(2 n ln 2 + 2) 2^-24, systematically only through c2 (half of that).  Sums of
many terms average the rest; the terms that carry a sum lie within 2^-24 of its
largest, which bounds the logarithm of a sum of them by
(24 ln 2 + 2) 2^-24 = 1.1e-6.
"""
import numpy as np

LOG_SUM = 1.2e-6


def bf16_bits(x):
    """Nearest-even bf16 patterns of float32 values."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    out = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    nan = np.where(np.signbit(x), np.uint16(0xFFC0), np.uint16(0x7FC0))
    return np.where(np.isnan(x), nan, out)


def as_dtype(x, dtype):
    return bf16_bits(x) if dtype == "bf16" else np.ascontiguousarray(x, np.float32)


def rows(kind, N, V, seed, dtype="f32"):
    """N rows of V float32 logits of one kind."""
    g = np.random.default_rng(seed)
    x = g.normal(0, 3, (N, V)).astype(np.float32)
    if kind == "ties":
        x = np.round(x / 2) * 2
    elif kind == "equal":
        x[:] = -1.5
    elif kind == "zeros":  # of both signs
        x = np.where(g.random((N, V)) < 0.5, np.float32(0.0), np.float32(-0.0))
    elif kind == "lowest":  # the type's lowest value everywhere
        x[:] = lowest(dtype)
    elif kind == "masked":  # few tokens left; one row none but one
        x[g.random((N, V)) < 0.97] = -np.inf
        x[:, V // 2] = 0.25
        x[0] = -np.inf
        x[0, V - 1] = 1.0
    elif kind == "masked_lowest":
        x[g.random((N, V)) < 0.9] = lowest(dtype)
        x[:, V // 3] = 0.25
    elif kind == "ascending":
        x = np.sort(x, -1)
    elif kind == "descending":
        x = -np.sort(-x, -1)
    elif kind == "block":  # the largest ones side by side
        n = min(V, 1500)
        x[:, :n] += 40.0
    elif kind == "peak":
        x[:, V // 2] += 60.0
    elif kind == "wide":
        x *= 1e4
    elif kind == "bad":
        x[0, V // 2] = np.nan
        if N > 1:
            x[1] = -np.inf
        if N > 2:
            x[2, V - 1] = np.inf
        if N > 3:  # a NaN with the sign set
            x[3, 0] = np.array(0xFFC00000, np.uint32).view(np.float32)
    elif kind != "normal":
        raise ValueError(kind)
    return x.astype(np.float32)


def lowest(dtype):
    return np.float32(-3.3895314e38) if dtype == "bf16" else np.finfo(np.float32).min


def uniforms(shape, seed):
    return (np.random.default_rng(seed).integers(0, 1 << 24, shape) / np.float32(1 << 24)).astype(np.float32)
