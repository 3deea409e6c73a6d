"""How far sums over many rows may be off in the operators around the packed attention, where their terms have either sign.

A sum of N such terms grows with the root of N, and a bound by the terms' magnitudes added up would let whole sequences be
missing.  Errors that do not depend on one another add up in squares too.

heads     dw of the head norms.  A term's error is at most e of its magnitude (e as for dx: (2 D + 32) 2^-24 + 2^-19), an addition's
          2^-24 of the sum so far, which is of the size of R, the root of the terms' squares: e R and sqrt(N) 2^-24 R, each at
          most a standard deviation; four and six of them.
experts   dw of the expert products, in the norm over an expert's elements.
          float32: sqrt(N) 2^-24, as above (and 16 2^-24 for the join of the parts).
          bfloat16: the tensor cores add 16 products at a time and cut off what has no place, half a step of 2^-23 of the sum's
          power of two on average, 0.36 2^-23 of the sum; 32 times until the sum goes to a register, and as the sum grows
          with the root of its terms it has two thirds of its last size on average: 32 x 0.36 x 2/3 x 2^-23 = 9.2e-7.  Twice that.
"""
import numpy as np

EXPERTS_BF16 = 2 * 32 * 0.36 * (2.0 / 3.0) * 2.0 ** -23


def heads(mag_terms):
    """A bound for each column, from the magnitudes of the terms [tokens, heads, D]."""
    n, h, D = mag_terms.shape
    e = (2 * D + 32) * 2.0 ** -24 + 2.0 ** -19
    return (4 * e + 6 * np.sqrt(n * h) * 2.0 ** -24) * np.sqrt((mag_terms ** 2).sum(axis=(0, 1)))


def experts(rows, bf16):
    """Of an expert with that many rows, relative to the norm of its gradient."""
    return EXPERTS_BF16 if bf16 else (np.sqrt(rows) + 16) * 2.0 ** -24
