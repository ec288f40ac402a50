"""What a softmax weight and its quotient may be off by where the scores are exact: each term a count of half steps u = 2^-24 of 32 bits."""
import numpy as np

U = 2.0 ** -24
F32, F16, BF16 = 0, 1, 2


def weight_bound(dtype):
    """Scores q K with one channel are exact, the largest is zero and the others' exponents s log2(e) / sqrt(d) are in [-2, 0]: the exponent's
    rounding (in fp16 weights are relative to 2^13, so of a number below 16: 8 u, else 2 u at most; ln 2 of it), the factor's (u of at most 2),
    the exponential (2 u), and what is left after the parts a weight enters the second product in (two of fp16: 2^-22, three of bf16: 2^-24)."""
    rounding = (8 if dtype == F16 else 2) * np.log(2) * U + 2 * np.log(2) * U + 2 * U
    return rounding + {F32: 0.0, F16: 4 * U, BF16: U}[dtype]


def quotient_bound(dtype, chain):
    """A sum of weights over the sum of all: both of them, `chain` additions each, the reciprocal and the product."""
    return 2 * weight_bound(dtype) + (2 * chain + 3) * U


def round_to(x, dtype):
    if dtype == F16:
        return x.astype(np.float16).astype(np.float32)
    bits = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return (((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def in_parts(w, dtype, parts):
    """Weights as the sum of `parts` numbers of the type, each the rounding of what the ones before it left; relative to 2^13 in fp16."""
    shift = np.float32(2.0 ** 13 if dtype == F16 else 1.0)
    rest, total = (w * shift).astype(np.float32), np.zeros(w.shape, np.float64)
    for _ in range(parts):
        p = round_to(rest, dtype)
        total += p
        rest = (rest - p).astype(np.float32)
    return total / shift


def grid_scores(g, heads, n):
    """q [heads], k [n]: powers of two and multiples of 1/16 that every type holds, the largest product zero, exponents down to -2 for d = 64."""
    q = np.array([1.0, 0.5, 0.25, 1.0])[np.arange(heads) % 4].astype(np.float32)
    k = -(g.integers(0, 177, n) / 16.0).astype(np.float32)
    k[g.integers(0, n)] = 0.0
    return q, k
