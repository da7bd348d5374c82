"""Plain-definition oracle of the linear layers on codes (numpy, 64 bits, CPU).  Test infrastructure, not product code.

* ``sums``      - exact products of code matrices (whole numbers below 2^53 in doubles).
* ``floats``    - the epilogue in doubles, and a bound on what its evaluation in 32 bits may be off by.
* ``codes``     - requantised sums, through the definition in ``direct.requant``.
* ``quantize``  - codes and scales of rows of floats.
"""
from __future__ import annotations

import math

import numpy as np

from . import direct

NONE, RELU, SILU, GELU = range(4)
U32 = 2.0 ** -24                     # half a step of a 32-bit float, relative


def sums(x: np.ndarray, w: np.ndarray) -> np.ndarray:
    """x [M, K] and w [N, K] code values -> int64 [M, N]."""
    t = np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T
    return t.astype(np.int64)


def codes(s: np.ndarray, bias, shift: int, lo: int, hi: int) -> np.ndarray:
    return direct.requant(s if bias is None else s + np.asarray(bias, dtype=np.int64), shift, lo, hi)


def _activate(v: np.ndarray, act: int) -> np.ndarray:
    if act == RELU:
        return np.maximum(v, 0.0)
    if act == SILU:
        return v / (1.0 + np.exp(-v))
    if act == GELU:
        return 0.5 * v * np.vectorize(math.erfc, otypes=[float])(-v * math.sqrt(0.5)) if v.size else v
    return v


def floats(s, x_scale=None, w_scale=None, bias=None, act=NONE, residual=None):
    """(value, bound): act(s x_scale[m] w_scale[n] + bias[n]) + residual in doubles, and how far 32-bit arithmetic in that order
    may be from it before the last rounding to the output's type.

    The sum becomes a float (half a step), is multiplied by x_scale (half a step) and goes with w_scale and bias into one fused
    multiply-add (half a step of its result): 2 U |product| + U |v|.  The activations' slopes stay below 1.13.  SILU adds an
    exponential of 2 ulp, a product, a sum and a quotient rounded to nearest: (4 + 1 + 1 + 1) U relative.  GELU: its argument is off by two half steps, where
    the slope of erf times the argument is below 0.5, erf by 2 ulp of at most 1, the sum by U of at most 2, then two products:
    (1 + 4 + 2) U |v| / 2 + 2 U |value|.  The residual's sum adds U |result|."""
    prod = np.asarray(s, dtype=np.float64)
    if x_scale is not None:
        prod = prod * np.asarray(x_scale, dtype=np.float64)[:, None]
    if w_scale is not None:
        prod = prod * np.asarray(w_scale, dtype=np.float64)
    v = prod if bias is None else prod + np.asarray(bias, dtype=np.float64)
    y = _activate(v, act)
    bound = 1.13 * (2 * U32 * np.abs(prod) + U32 * np.abs(v))
    if act == SILU:
        bound = bound + 7 * U32 * np.abs(y)
    elif act == GELU:
        bound = bound + 3.5 * U32 * np.abs(v) + 2 * U32 * np.abs(y)
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
        bound = bound + U32 * np.abs(y)
    return y, bound * 1.01 + 2.0 ** -126         # products of the half steps; results in the subnormal range


def quantize(x: np.ndarray, bits: int, signed: bool):
    """Codes (int64) and scales (float32) of the rows of x, which holds float32, float16 or bfloat16 values in any wider type.

    The definition divides in 32 bits; a quotient of two floats rounded to 64 and then to 32 bits is the one rounded to 32."""
    v = np.asarray(x, dtype=np.float64)
    hi = (1 << (bits - 1)) - 1 if signed else (1 << bits) - 1
    lo = -(1 << (bits - 1)) if signed else 0
    with np.errstate(all="ignore"):
        top = np.abs(v).max(axis=1) if signed else np.maximum(v.max(axis=1), 0.0)
        scale = (top / hi).astype(np.float32)
        quot = (v / scale.astype(np.float64)[:, None]).astype(np.float32)
        c = np.clip(np.rint(quot.astype(np.float64)), lo, hi)
    return np.where(np.isnan(c), 0, c).astype(np.int64), scale
