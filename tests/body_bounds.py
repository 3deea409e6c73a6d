"""How far the gradients of packed attention may be off, from the arithmetic of the kernels.

The gradients' definition takes the stored out and lse, so their rounding is no error here.  With e_S the relative
error of P = exp(scale S - lse), |scale S| <= Z = max |scale q| |k|, and sums in 32 bits (a step of 2^-23 a term,
twice half a step, since tensor cores may cut off what they add):
  S         D products: D Z 2^-23 in the exponent; the scale times log2 e, its product and the difference with lse:
            three roundings of Z and of |lse|: (3 Z + 4 |lse|) 2^-23;  the exponential itself 2^-21
  dP, delta D products each, of magnitudes that "parts_" sums: c = (D + 8) 2^-23 of it
  dS        |dS| e_S, and rounded for the second product: u = 2^-8 in bfloat16, nothing in float32
  sums      N terms (the keys, or the queries of all heads of a group): (N + 16) 2^-23 of "terms_"
  result    u |value|, half a step of its type
``element`` adds all of them up at their largest.  ``norm`` bounds the Frobenius norm of a gradient's error, where the
roundings of many elements, each anywhere within its half step, add up in squares: a third of u^2 for each
term and each result; the 32-bit errors of S by sqrt(D) for D; those that a whole row shares (lse) and
the parts at their largest.  A quarter more for the draw: with the thousands of elements that it is used for, the
sum of squares is within a few per cent of its mean.
"""
import numpy as np


def _setting(q, k, lse, cu, scale, bf16):
    D, g = q.shape[2], q.shape[1] // k.shape[1]
    Z = abs(scale) * np.linalg.norm(q, axis=2).max() * np.linalg.norm(k, axis=2).max()
    L, longest = np.abs(lse).max(), int(np.diff(cu).max())
    return D, Z, L, {"dq": longest, "dk": longest * g, "dv": longest * g}, (2.0 ** -8 if bf16 else 0.0), 2.0 ** -8 if bf16 else 2.0 ** -24


def element(name, ref, q, k, lse, cu, scale, bf16):
    """Bound of |error| for every element of gradient `name`; `ref` is the float64 form's dict."""
    D, Z, L, N, second, u = _setting(q, k, lse, cu, scale, bf16)
    e = (D * Z + 3 * Z + 4 * L) * 2.0 ** -23 + 2.0 ** -21
    return (u * np.abs(ref[name]) + 1.01 * ((second + e + (N[name] + 16) * 2.0 ** -23) * ref["terms_" + name]
                                            + (D + 8) * 2.0 ** -23 * ref["parts_" + name]))


def norm(name, ref, q, k, lse, cu, scale, bf16):
    """Bound of the error's Frobenius norm."""
    D, Z, L, N, second, u = _setting(q, k, lse, cu, scale, bf16)
    e = (np.sqrt(D) + 3) * Z * 2.0 ** -23 + 2.0 ** -21
    one, terms = np.linalg.norm(ref[name]), np.sqrt(ref["squares_" + name].sum())
    random = np.sqrt(u * u / 3 * one ** 2 + (second ** 2 / 3 + e * e) * terms ** 2)
    return 1.25 * random + (4 * L + np.sqrt(N[name]) + 16) * 2.0 ** -23 * one + (np.sqrt(D) + 8) * 2.0 ** -23 * np.linalg.norm(
        ref["parts_" + name])
