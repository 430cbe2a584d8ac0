"""Attention over the paged store where value rows differ much in size, and how many bits its
weights keep: every bound is relative to what the row itself sums up (tests/weighted.py)."""
import math

import numpy as np
import pytest
import torch

import drafts
import weighted
from drafts import PAGE, randn
from paper_2608_21541_gb300 import certkv as ck

pytestmark = pytest.mark.gpu


def check(out, lse, q, store, n, k_new=None, v_new=None):
    """q [1][1][T][G][128] over one segment of n slots (and drafts under the chain mask)."""
    T, G = q.shape[2], q.shape[3]
    at = drafts.slots(store.table.cpu().numpy(), 0, 0, n)
    K, V = (drafts.values({a: b[at] for a, b in drafts.held(store, x).items()}) for x in "kv")
    for t in range(T):
        Kt, Vt = K, V
        if k_new is not None:
            new = [x[0, 0, :t + 1, 0].double().cpu().numpy() for x in (k_new, v_new)]
            Kt, Vt = np.concatenate([K, new[0]]), np.concatenate([V, new[1]])
        qs = q[0, 0, t].double().cpu().numpy()
        o, tol, e, etol = weighted.attention(qs, Kt, Vt, store.format)
        got = out[0, 0, t].double().cpu().numpy()
        assert np.isfinite(got).all()
        d = np.abs(got - o)
        assert (d <= tol).all(), (t, np.max(d / tol), np.max(d) / np.max(np.abs(o)))
        assert (np.abs(lse[0, 0, t].double().cpu().numpy() - e) <= etol).all()


def run(fmt, k, v, q, k_new=None, v_new=None):
    n = k.shape[2]
    st = ck.Store.empty(1, -(-n // PAGE), fmt)
    g = torch.Generator().manual_seed(n)
    st.table.copy_(torch.randperm(st.table.numel(), generator=g).view(1, -1))
    ck.certkv_store_append(k, v, st)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = ck.certkv_tree_attn(q, st, hkv=1, k_new=k_new, v_new=v_new, lse=lse)
    assert st.read_status() == 0
    check(out, lse, q, st, n, k_new, v_new)
    return out


def inputs(T, G, n, size, seed, sink=None, bits=0.0):
    """q, k, v; base-2 logits spread by a few bits, values of `size`, and slot `sink`'s logit
    `bits` above (or below) nought for every row."""
    q, k = randn((1, 1, T, G, 128), seed), randn((1, 1, n, 1, 128), seed + 1, gain=0.5)
    v = (randn((1, 1, n, 1, 128), seed + 2).float() * size).bfloat16()
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    if sink is not None:
        k[0, 0, sink] = 0.0
        k[0, 0, sink, 0, 0] = bits * math.log(2.0) * math.sqrt(128) / 8.0
    return q, k, v


# query rows: few (mma.sync; over a bf16 store 24 are for tcgen05), up to 128, more
ROWS = [(1, 4), (3, 8), (16, 4), (9, 16)]


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G", ROWS)
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-6])
@pytest.mark.parametrize("sink", [0, 70, 1400])
def test_zero_value_row_with_a_large_weight(fmt, T, G, size, sink):
    """An attention sink: a key that takes most of every row's weight, whose value is zero."""
    q, k, v = inputs(T, G, 1501, size, 300, sink, 14.0)
    v[0, 0, sink] = 0.0
    run(fmt, k, v, q)
    v[0, 0, sink] = -0.0
    v[0, 0, sink + 1:sink + 90] = 0.0  # and a whole tile of them
    run(fmt, k, v, q)


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G", ROWS)
@pytest.mark.parametrize("slot", [0, 64, 1000])
@pytest.mark.parametrize("larger", [2.0 ** 20, 2.0 ** 60, 2.0 ** -40])
def test_value_row_of_another_size_with_a_small_weight(fmt, T, G, slot, larger):
    """One value row 2^20 (2^60) times the others, seen with 2^-40 (2^-80) of their weight, and
    a small row seen with nearly all of it."""
    bits = -2.0 * math.log2(larger) if larger > 1.0 else 20.0
    q, k, v = inputs(T, G, 1201, 1.0, 310, slot, bits)
    v[0, 0, slot] *= larger
    run(fmt, k, v, q)


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G", ROWS)
def test_all_values_zero(fmt, T, G):
    q, k, v = inputs(T, G, 200, 0.0, 320)
    assert not run(fmt, k, v, q).float().any()


@pytest.mark.parametrize("fmt,top", [("fp8", 448.0), ("fp4", 2688.0)])
@pytest.mark.parametrize("T,G", ROWS)
def test_rows_whose_scale_is_one(fmt, top, T, G):
    """Rows held with the scale that zero rows have, among rows of zeros: one element alone, at
    either end, counts."""
    q, k, v = inputs(T, G, 300, 1.0, 330)
    v[0, 0, ::3] = 0.0
    for i, d in enumerate((0, 15, 16, 63, 64, 127)):
        v[0, 0, 3 * i] = 0.0
        v[0, 0, 3 * i, 0, d] = -top if i % 2 else top
    run(fmt, k, v, q)


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G", ROWS)
def test_drafts_of_another_size(fmt, T, G):
    """Drafts' own values far above and below the store's, and zero."""
    q, k, v = inputs(T, G, 700, 1e-2, 340)
    kn, vn = randn((1, 1, T, 1, 128), 343, gain=0.5), randn((1, 1, T, 1, 128), 344)
    for i in range(T):
        vn[0, 0, i] *= (0.0, 1e-6, 1e3, 1.0)[i % 4]
    run(fmt, k, v, q, kn, vn)


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G", ROWS)
def test_weights_keep_their_bits_where_values_cancel(fmt, T, G):
    """Slots in pairs of nearly the same weight and opposite values: the result is 2^-8 of what
    is summed, so a weight's rounding shows undiminished by the result's own."""
    n = 256
    q, k, v = inputs(T, G, n, 1.0, 350)
    q[..., 1:] *= 0.125
    k[0, 0, 1::2] = k[0, 0, ::2]
    k[0, 0, 1::2, 0, 0] += 2.0 ** -8  # logit 2^-8 / sqrt(2) higher
    v[0, 0, ::2] = randn((1, 1, 128), 353).sign()
    v[0, 0, 1::2] = -v[0, 0, ::2]
    run(fmt, k, v, q)


@pytest.mark.parametrize("fmt", ("bf16", "fp8", "fp4"))
@pytest.mark.parametrize("T,G,n", [(1, 4, 20011), (3, 8, 9001), (16, 4, 20011), (9, 16, 9001)])
def test_long_segments(fmt, T, G, n):
    q, k, v = inputs(T, G, n, 1.0, 360)
    run(fmt, k, v, q)
