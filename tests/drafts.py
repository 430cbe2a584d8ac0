"""Plain 64-bit definitions of the operators on drafted tokens (rotary positions,
the paged store, tree attention), and the small inputs their tests share."""
import math

import numpy as np
import torch

PAGE, D = 64, 128
ROW = {"bf16": 256, "fp8": 128, "fp4": 64}


def grid(man, low, top):
    """Non-negative values of a small float: `man` mantissa bits, smallest normal
    exponent `low`, largest value `top`."""
    vals = [m * 2.0 ** (low - man) for m in range(2 ** man)]
    e = low
    while vals[-1] < top:
        vals += [(2 ** man + m) * 2.0 ** (e - man) for m in range(2 ** man)]
        e += 1
    return np.array([v for v in vals if v <= top])


E4M3, E2M1 = grid(3, -6, 448.0), grid(1, 0, 6.0)


def nearest(y, g):
    """Index and value of the grid entry nearest to |y| (ties to the even index,
    which is the even mantissa; beyond the largest: the largest), with y's sign."""
    a = np.abs(y.astype(np.float64))
    hi = np.clip(np.searchsorted(g, a), 1, len(g) - 1)
    lo = hi - 1
    dl, dh = a - g[lo], g[hi] - a
    idx = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return idx, np.where(np.signbit(y), -g[idx], g[idx])


def encode(rows, fmt):
    """What a store holds for bf16 rows [n][128]: dict of values the codes stand for
    before the row scale ("codes"), "group" (fp4) and "scale"; fp32 steps as
    the store's definition has them."""
    x = rows.float().numpy()
    if fmt == "bf16":
        return {"codes": x, "scale": np.ones(len(x), np.float32)}
    top = np.float32(448.0 if fmt == "fp8" else 2688.0)
    one = np.float32(1.0)
    A = np.abs(x).max(1)
    bad = ~np.isfinite(x).all(1)
    small = (A < np.float32(2.0 ** -100)) | bad
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        s = np.where(bad, np.nan, np.where(small, one, A * (one / top))).astype(np.float32)
        r = np.where(small, np.float32(0), (one / A) * top).astype(np.float32)
    xs = np.where(bad[:, None], np.float32(0), x)
    if fmt == "fp8":
        return {"codes": nearest(xs * r[:, None], E4M3)[1], "scale": s}
    g = xs.reshape(-1, 8, 16)
    gs = nearest((np.abs(g).max(2) * r[:, None]) * (one / np.float32(6)), E4M3)[1]
    gs = gs.astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        m = np.where(gs > 0, r[:, None] * (one / gs), np.float32(0)).astype(np.float32)
    codes = nearest(g * m[:, :, None], E2M1)[1]
    return {"codes": codes.reshape(-1, D), "group": gs, "scale": s}


def values(enc):
    """The rows an encoding stands for, in 64 bits."""
    c = enc["codes"].astype(np.float64)
    if "group" in enc:
        c = c * np.repeat(enc["group"].astype(np.float64), 16, axis=1)
    return c * enc["scale"].astype(np.float64)[:, None]


def held(store, name):
    """Codes (as values), group scales and scales a Store's pool holds, flat over slots."""
    raw = getattr(store, name).contiguous().view(torch.uint8).cpu().numpy()
    n = raw.shape[0] * PAGE
    raw = raw.reshape(n, -1)
    if store.format == "bf16":
        x = torch.from_numpy(raw.copy()).view(torch.bfloat16).float().numpy()
        return {"codes": x, "scale": np.ones(n, np.float32)}
    scale = getattr(store, name + "_scale").cpu().numpy().reshape(n)
    if store.format == "fp8":
        return {"codes": fp8(raw), "scale": scale}
    grp = getattr(store, name + "_group").contiguous().view(torch.uint8).cpu().numpy()
    nib = np.stack([raw & 15, raw >> 4], -1).reshape(n, D)
    val = E2M1[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    return {"codes": val, "group": fp8(grp.reshape(n, 8)).astype(np.float32), "scale": scale}


def fp8(raw):
    v = np.concatenate([E4M3, [np.nan]])[raw & 127]
    return np.where(raw & 128, -v, v)


def slots(table, u, first, n):
    """Pool slots of slots first .. first + n - 1 of segment u (-1: no page)."""
    s = first + np.arange(n)
    page = table[u, s // PAGE]
    return np.where(page < 0, -1, page.astype(np.int64) * PAGE + s % PAGE)


def visible(mask, b, t, T):
    """The drafts token t of sequence b sees."""
    if mask is None:
        return list(range(t + 1))
    w = int(mask[b, t])
    return [j for j in range(T) if w >> j & 1]


def attention(q, store, counts, hkv, k_new=None, v_new=None, mask=None, scale=None):
    """(out, lse, vmax, mag) in 64 bits: the operator's definition.  vmax: the largest
    |v| element a row can draw on; mag: the largest scale * sum_i |q_i k_i|."""
    q = q.float().cpu().numpy().astype(np.float64)
    B, L, T, Hq, _ = q.shape
    G = Hq // hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    kv = [values(held(store, "k")), values(held(store, "v"))]
    table = store.table.cpu().numpy()
    new = [None, None] if k_new is None else [x.float().cpu().numpy().astype(np.float64)
                                              for x in (k_new, v_new)]
    mask = None if mask is None else mask.cpu().numpy()
    out = np.zeros(q.shape)
    lse = np.full(q.shape[:-1], -np.inf)
    vmax, mag = np.zeros(lse.shape), np.zeros(lse.shape)
    for b in range(B):
        for l in range(L):
            for h in range(hkv):
                u = (b * L + l) * hkv + h
                at = slots(table, u, 0, counts[u])
                at = at[at >= 0]
                for t in range(T):
                    K, V = kv[0][at], kv[1][at]
                    if new[0] is not None:
                        see = visible(mask, b, t, T)
                        K = np.concatenate([K, new[0][b, l, see, h]])
                        V = np.concatenate([V, new[1][b, l, see, h]])
                    if not len(K):
                        continue
                    qs = q[b, l, t, h * G:(h + 1) * G]
                    with np.errstate(invalid="ignore", over="ignore"):
                        x = scale * (qs @ K.T)
                        m = x.max(1, keepdims=True)
                        p = np.exp(x - m)
                        o = (p @ V) / p.sum(1, keepdims=True)
                        e = m[:, 0] + np.log(p.sum(1))
                    sl = np.s_[b, l, t, h * G:(h + 1) * G]
                    out[sl], lse[sl] = o, e
                    vmax[sl] = np.abs(V).max()
                    mag[sl] = scale * (np.abs(qs) @ np.abs(K).T).max(1)
    return out, lse, vmax, mag


def check_attention(out, lse, ref):
    """bf16 rounding of the output (half an ulp, 2^-8 of it) plus weights and a normaliser
    held to 2^-9 of the largest value each; the log-sum-exp to the fp32 accumulation of
    128 products (128 2^-23 of their magnitudes' sum)."""
    o, e, vmax, mag = ref
    got = out.float().cpu().numpy()
    assert np.isfinite(got).all()
    tol = 2.0 ** -8 * np.abs(o) + 2.0 ** -8 * vmax[..., None] + 1e-30
    assert (np.abs(got - o) <= tol).all(), np.max(np.abs(got - o) / tol)
    if lse is not None:
        g = lse.cpu().numpy()
        fin = np.isfinite(e)
        np.testing.assert_array_equal(g[~fin], e[~fin])
        tol = 1e-5 + 2.0 ** -16 * mag[fin] + 2.0 ** -20 * np.abs(e[fin])
        assert (np.abs(g[fin] - e[fin]) <= tol).all(), np.max(np.abs(g[fin] - e[fin]) / tol)


def random_tree(T, rng):
    """int64 words [T]: every token sees itself and its ancestors."""
    seen = []
    for i in range(T):
        p = int(rng.integers(-1, i)) if i else -1
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    return [w - (1 << 64) if w >= 1 << 63 else w for w in seen]


def randn(shape, seed, device="cuda", gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(torch.bfloat16).to(device)
