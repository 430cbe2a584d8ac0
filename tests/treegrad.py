"""The gradients of tree attention over a paged store in 64 bits, and how far a kernel may be
from them: the definitions of include/certkv.h on the values that the store holds."""
import math

import numpy as np
import torch

import drafts
from drafts import D


def gradients(q, store, counts, hkv, out, lse, dout, k_new=None, v_new=None, mask=None, scale=None,
              dlse=None):
    """{name: (value, tolerance)}: dq [B][L][T][Hq][D], dk, dv [B][L][T][H][D] and dk_store,
    dv_store [pool slots][D] (NaN where no live slot is).

    Tolerance of an element, as the sum of |terms| with these relative errors:
      2^-8 of the result: its rounding to bf16;
      2^-14 of each p or e: a matrix operand in two bf16 parts, either cut off at 8 bits, which
        leaves 2^-7 of what it stands for;
      of each p 2^-15 mag + 2^-15, mag = scale sum |q k| + |lse|: a logit is an fp32 sum of 128
        products (128 2^-24 of their magnitudes' sum) times a rounded scale less an fp32 lse, and
        the hardware exponential is off by 2^-22;
      of each <dout, v> - delta 2^-16 of the sum of the products' magnitudes: fp32 sums."""
    f = lambda x: x.float().cpu().numpy().astype(np.float64)  # noqa: E731
    q, out, dout, lse = f(q), f(out), f(dout), f(lse)
    B, L, T, Hq, _ = q.shape
    G = Hq // hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    kv = [drafts.values(drafts.held(store, "k")), drafts.values(drafts.held(store, "v"))]
    table = store.table.cpu().numpy()
    new = None if k_new is None else [f(k_new), f(v_new)]
    mask = None if mask is None else mask.cpu().numpy()
    dl = np.zeros(lse.shape) if dlse is None else f(dlse)
    res = {"dq": q.shape}
    if new is not None:
        res.update(dk=new[0].shape, dv=new[0].shape)
    res = {n: (np.zeros(s), np.zeros(s)) for n, s in res.items()}
    pool = (len(kv[0]), D)
    for n in ("dk_store", "dv_store"):
        res[n] = (np.full(pool, np.nan), np.zeros(pool))
    U, P = 2.0 ** -8, 2.0 ** -14
    for b in range(B):
        see = np.zeros((T, T), bool)
        for t in range(T):
            see[t, drafts.visible(mask, b, t, T)] = True
        for l in range(L):
            for h in range(hkv):
                u = (b * L + l) * hkv + h
                at = drafts.slots(table, u, 0, counts[u])
                at = at[(at >= 0) & (at < len(kv[0]))]
                n = len(at)
                K, V = kv[0][at], kv[1][at]
                live = np.ones((T, G, n), bool)
                if new is not None:
                    K = np.concatenate([K, new[0][b, l, :, h]])
                    V = np.concatenate([V, new[1][b, l, :, h]])
                    live = np.concatenate([live, np.broadcast_to(see[:, None], (T, G, T))], 2)
                sl = np.s_[b, l, :, h * G:(h + 1) * G]
                R = T * G
                Q, O, DO = (x[sl].reshape(R, D) for x in (q, out, dout))
                lr, dr = lse[sl].reshape(R, 1), dl[sl].reshape(R, 1)
                live = live.reshape(R, -1) & (lr > -np.inf)
                Kf, Vf = (np.where(np.isfinite(x), x, 0) for x in (K, V))
                Qf, DOf = (np.where(lr > -np.inf, x, 0) for x in (Q, DO))
                x = scale * (Qf @ Kf.T)
                with np.errstate(over="ignore", invalid="ignore"):
                    p = np.where(live, np.exp(np.where(live, x - lr, 0)), 0)
                    mag = scale * (np.abs(Qf) @ np.abs(Kf).T) + np.where(lr > -np.inf, np.abs(lr), 0)
                pull = DOf @ Vf.T - (DOf * np.where(lr > -np.inf, O, 0)).sum(1, keepdims=True) + dr
                amag = np.abs(DOf) @ np.abs(Vf).T + (np.abs(DOf) * np.abs(O)).sum(1, keepdims=True) \
                    + np.abs(dr)
                e = scale * p * pull
                rel = 2.0 ** -15 * (mag + 1)
                pe = p * (P + rel)
                ee = np.abs(e) * (P + rel) + scale * p * 2.0 ** -16 * amag
                dq = e @ Kf
                res["dq"][0][sl] = dq.reshape(T, G, D)
                res["dq"][1][sl] = (U * np.abs(dq) + ee @ np.abs(Kf)).reshape(T, G, D)
                dk, dv = e.T @ Qf, p.T @ DOf
                tk, tv = U * np.abs(dk) + ee.T @ np.abs(Qf), U * np.abs(dv) + pe.T @ np.abs(DOf)
                for name, x, tol in (("dk", dk, tk), ("dv", dv, tv)):
                    if new is not None:
                        res[name][0][b, l, :, h], res[name][1][b, l, :, h] = x[n:], tol[n:]
                    res[name + "_store"][0][at], res[name + "_store"][1][at] = x[:n], tol[:n]
    return res


def check(got, ref, name):
    want, tol = ref[name]
    got = got.float().cpu().numpy().reshape(want.shape)
    live = ~np.isnan(want)
    assert np.isfinite(got[live]).all(), name
    worst = np.abs(got - want)[live] / (tol[live] + 1e-30)
    assert worst.size == 0 or worst.max() <= 1, (name, worst.max())
