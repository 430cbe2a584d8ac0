"""The bound of tests/weighted.py on the CPU, against attention computed with the roundings it
states, and with planted mistakes that it has to see: a weight's bf16 remainder left out, a
tile's values taken in another order."""
import math

import numpy as np
import pytest
import torch

import weighted


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def cancelling(seed, n=256):
    """Slots in pairs of nearly the same weight and opposite values."""
    g = np.random.default_rng(seed)
    q, K = bf16(g.standard_normal((4, 128))), bf16(0.5 * g.standard_normal((n, 128)))
    q[:, 1:] *= 0.125
    q[:, 0], K[:, 0] = 8.0, 0.0
    K[1::2] = K[::2]
    K[1::2, 0] += 2.0 ** -8
    V = np.empty((n, 128))
    V[::2] = np.sign(g.standard_normal(128))
    V[1::2] = -V[::2]
    return q, K, V


def result(q, K, V, parts):
    x = q @ K.T / math.sqrt(128)
    w = np.exp(x - x.max(1, keepdims=True))
    hi = bf16(w)
    used = hi + bf16(w - hi) if parts == 2 else hi
    return bf16(used @ V / w.sum(1, keepdims=True))


@pytest.mark.parametrize("seed", range(4))
def test_a_weight_without_its_remainder_is_seen(seed):
    q, K, V = cancelling(seed)
    o, tol, _, _ = weighted.attention(q, K, V, "bf16")
    assert (np.abs(result(q, K, V, 2) - o) <= tol).all()
    assert not (np.abs(result(q, K, V, 1) - o) <= tol).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
def test_a_tile_of_values_in_another_order_is_seen(fmt):
    g = np.random.default_rng(5)
    q, K, V = (bf16(g.standard_normal(s) * a) for s, a in (((4, 128), 1.0), ((20011, 128), 0.5),
                                                           ((20011, 128), 1.0)))
    o, tol, _, _ = weighted.attention(q, K, V, fmt)
    assert (np.abs(result(q, K, V, 2) - o) <= tol).all()
    V2 = V.copy()
    V2[1280:1408] = V[1280:1408][::-1]
    assert not (np.abs(result(q, K, V2, 2) - o) <= tol).all()
    V2[1280:1408] = 0.0
    assert not (np.abs(result(q, K, V2, 2) - o) <= tol).all()
