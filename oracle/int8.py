"""CPU oracle of the layer in 8-bit integers (csrc/moe_quant.hip, csrc/moe_ffn_i8.hip) -- TEST INFRASTRUCTURE ONLY, plain numpy.

    quantize    rows in 8 bits by the definition of include/moe.h, in float32 operation by operation: whole numbers and scales are exact
    product     sums of whole numbers, exact in doubles (below 2^53), times the scales of column and row
    gate_up     silu(g) * u of two such products, in doubles and not rounded, with the bound that a kernel's float32 arithmetic has to keep
    rmsnorm     residual and norm in doubles, with such a bound
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                                   # half a step of float32, relative
U16 = 2.0 ** -8                                  # half a step of bf16, relative


def quantize(v: np.ndarray):
    """float32 [T, N] -> (int8 [T, N], float32 [T])."""
    v = np.asarray(v, dtype=np.float32)
    most = np.abs(v).max(axis=1)
    bad = ~np.isfinite(v).all(axis=1)
    with np.errstate(all="ignore"):
        scale = np.maximum(most / np.float32(127), np.float32(2.0 ** -126))
        inverse = np.minimum(np.float32(127) / most, np.float32(2.0 ** 126))
        q = np.rint(np.where(bad[:, None], np.float32(0), v * inverse[:, None]))
    scale[bad] = np.nan
    assert np.abs(q).max(initial=0) <= 127
    return q.astype(np.int8), scale


def product(x_q, x_scale, W, w_scale) -> np.ndarray:
    """[T, K], [T], [N, K], [N] -> float64 [T, N]; a kernel converts the sum (U), multiplies twice (2 U)."""
    return (x_q.astype(np.float64) @ W.astype(np.float64).T) * w_scale.astype(np.float64) * x_scale.astype(np.float64)[:, None]


PRODUCT = 3.001 * U                              # relative error of a float32 product


def gate_up(x_q, x_scale, W1, w1, W3, w3):
    """-> (h float64, bound on a kernel's error before it rounds h to bf16).  g and u are off by PRODUCT.  e = 2^(-g log2 e): its exponent is off by
    (PRODUCT + 2 U) |g| log2 e in the exponent, |g| (PRODUCT + 2 U) relative, and the hardware's exp2 and reciprocal by a unit in the last place
    (2 U) each; the sum, the two products by U."""
    g, u = product(x_q, x_scale, W1, w1), product(x_q, x_scale, W3, w3)
    with np.errstate(over="ignore"):
        h = g / (1.0 + np.exp(-g)) * u
    rel = np.abs(g) * (PRODUCT + 2 * U) + 2 * PRODUCT + 8 * U
    return h, np.abs(h) * rel + 2.0 ** -126


def rmsnorm(hidden, delta, gamma, eps: float):
    """-> (s, y, relative bound on y).  s = hidden + delta rounded to float32 as the kernel holds it; a sum of n squares taken 32 to a thread and then in a tree
    is off by (32 + 10) U relative, half of that under the root; root, reciprocal, mean and two products 6 U."""
    s = np.asarray(delta, np.float32) if hidden is None else np.asarray(hidden, np.float32) + np.asarray(delta, np.float32)
    d = s.astype(np.float64)
    y = d / np.sqrt(np.mean(d * d, axis=1, keepdims=True) + eps) * np.asarray(gamma, np.float64)
    return s, y, 30 * U
