"""Attention in 64 bits with what a row sums up, S = sum_s p_s |v_s| of each element, and a bound
on the output relative to it:
  2^-8 |o|                 the bf16 result, half an ulp;
  S r                      a weight's rounding: 2^-16 over bf16 stores (two bf16 parts), 2^-11
                           over 8- and 4-bit ones (weight times value scale, once to f16);
  S 2 (2^-17 m + 2^-21 x)  the logits, as weights and in the normaliser: 128 fp32 products of
                           magnitudes m, scale and exponential of logits up to x;
  S (n / 16 + 64) 2^-23    fp32 additions of n slots, sixteen a product, and of records;
  n 2^-29 max p_s |v_s|    f16 weights below 2^-14: half of 2^-24 each, against a largest
                           of 2^5 times the reference."""
import math

import numpy as np

ROUNDING = {"bf16": 2.0 ** -16, "fp8": 2.0 ** -11, "fp4": 2.0 ** -11}


def attention(q, K, V, fmt):
    """(out, bound of out, log-sum-exp, bound of it) of rows q [R][128] over K, V [n][128]."""
    x = q @ K.T / math.sqrt(128)
    m = x.max(1, keepdims=True)
    p = np.exp(x - m)
    total = p.sum(1, keepdims=True)
    p /= total
    o, S = p @ V, p @ np.abs(V)
    mag = (np.abs(q) @ np.abs(K).T).max(1) / math.sqrt(128)
    d = 2.0 ** -17 * mag + 2.0 ** -21 * np.abs(x).max(1)
    rel = ROUNDING[fmt] + 2 * d + (len(K) / 16 + 64) * 2.0 ** -23
    top = (p * np.abs(V).max(1)).max(1)
    tol = 2.0 ** -8 * np.abs(o) + rel[:, None] * S + len(K) * 2.0 ** -29 * top[:, None] + 1e-38
    lse = m[:, 0] + np.log(total[:, 0])
    return o, tol, lse, 1e-5 + 2.0 ** -16 * mag + 2.0 ** -20 * np.abs(lse)
