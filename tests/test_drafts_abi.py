"""Refusals of the operators on drafted tokens: every argument is checked on the host
before anything is launched (CPU only; no call reaches a GPU)."""
import ctypes

import pytest
import torch

from paper_2608_21541_gb300 import build as B
from paper_2608_21541_gb300 import certkv as ck

FAKE = 1 << 20  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    B.build()
    return ck.load_library()


def rows(data=FAKE, sb=1 << 20, sl=1 << 18, st=1024, sh=128):
    return ck.certkv_rows(data, sb, sl, st, sh)


def store(**kw):
    f = dict(units=16, format=1, max_pages=4, pool_pages=64, k=FAKE, v=FAKE, k_group=None,
             v_group=None, k_scale=FAKE, v_scale=FAKE, table=FAKE, counts=FAKE, status=None)
    f.update(kw)
    return ck.certkv_store(*f.values())


BAD_STORES = [dict(units=0), dict(units=(1 << 24) + 1), dict(format=3), dict(format=-1),
              dict(max_pages=0), dict(max_pages=(1 << 18) + 1), dict(pool_pages=0),
              dict(pool_pages=1 << 25), dict(k=None), dict(v=FAKE + 64), dict(k_scale=None),
              dict(v_scale=FAKE + 4), dict(format=2), dict(format=2, k_group=FAKE, v_group=FAKE + 8),
              dict(table=None), dict(counts=None), dict(counts=FAKE + 2), dict(status=FAKE + 1)]


def test_rope_plan_refuses(lib):
    out = ck.certkv_rope_angles()

    def plan(dim=64, layout=0, base=1e4, sc=None):
        return lib.certkv_rope_plan(dim, layout, base, ctypes.byref(sc) if sc else None,
                                    ctypes.byref(out))

    sc = ck.certkv_rope_scaling
    assert plan() == ck.OK and out.dim == 64 and out.magnitude == 1.0
    for kw in (dict(dim=0), dict(dim=130), dict(dim=7), dict(layout=2), dict(base=1.0),
               dict(base=float("nan")), dict(sc=sc(4, 2, 1, 0, 1, 1)), dict(sc=sc(1, 0, 1, 0, 1, 1)),
               dict(sc=sc(1, 2, 1, 0, 1, 0)), dict(sc=sc(2, 2, 1, 0, 1, 1), dim=2),
               dict(sc=sc(3, 2, 0, 0, 1, 1)), dict(sc=sc(3, 2, 8192, 1, 1, 1)),
               dict(sc=sc(3, float("inf"), 8192, 0, 1, 1))):
        assert plan(**kw) == ck.EINVAL, kw
    assert lib.certkv_rope_plan(64, 0, 1e4, None, None) == ck.EINVAL
    with pytest.raises(ValueError):
        ck.certkv_rope_plan(64, layout="diagonal")
    with pytest.raises(ck.CertKVError):
        ck.certkv_rope_plan(63)


def test_rope_plan_holds_the_frequencies(lib):
    import math
    plan = ck.certkv_rope_plan(96, base=500000.0, scaling="ramp", factor=8.0, original=4096.0,
                               low=1.0, high=4.0, magnitude=1.25)
    for i in range(64):
        th = 500000.0 ** (-2.0 * i / 96)
        g = min(1.0, max(0.0, (4096 * th / (2 * math.pi) - 1.0) / 3.0))
        want = ((1 - g) * th / 8.0 + g * th) / (2 * math.pi) if i < 48 else 0.0
        assert abs(plan.turns_hi[i] + plan.turns_lo[i] - want) <= 2.0 ** -46 * want
    assert plan.magnitude == 1.25 and abs(plan.inverse_magnitude - 0.8) < 1e-7


def test_rope_refuses(lib):
    plan = ck.certkv_rope_plan(64)

    def call(b=2, l=2, t=4, hq=8, hkv=2, q=rows(), qo=rows(), k=None, ko=None, pos=FAKE, plan=plan,
             inv=0):
        ref = [ctypes.byref(x) if x is not None else None for x in (q, qo, k, ko)]
        return lib.certkv_rope(b, l, t, hq, hkv, *ref, pos, ctypes.byref(plan) if plan else None,
                               inv, None)

    bad = ck.certkv_rope_angles(dim=5)
    for kw in (dict(b=0), dict(l=0), dict(t=0), dict(hq=0), dict(hkv=-1), dict(q=None),
               dict(qo=None), dict(q=rows(FAKE + 8)), dict(q=rows(sh=132)), dict(k=rows()),
               dict(k=rows(), ko=rows(), hkv=0), dict(pos=None), dict(pos=FAKE + 2),
               dict(plan=None), dict(plan=bad), dict(inv=2), dict(qo=rows(sb=0)),
               dict(qo=rows(sh=64)), dict(qo=rows(st=512)), dict(b=1 << 20, t=1 << 20)):
        assert call(**kw) == ck.EINVAL, kw


@pytest.mark.parametrize("bad", BAD_STORES)
def test_store_refused_by_every_entry_point(lib, bad):
    st, r = store(**bad), rows()
    packed = ck.certkv_packed(FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30)
    shape = ck.certkv_shape(2, 4, 8, 2, 2, 128, 1)
    assert lib.certkv_store_load(ctypes.byref(packed), 1, 0, ctypes.byref(st), 256, 1 << 30,
                                 None) == ck.EINVAL
    assert lib.certkv_store_append(2, 4, 2, 3, ctypes.byref(r), ctypes.byref(r), None, None, None,
                                   ctypes.byref(st), None) == ck.EINVAL
    assert lib.certkv_store_read(ctypes.byref(st), None, 1, FAKE, FAKE, None) == ck.EINVAL
    assert lib.certkv_tree_attn(ctypes.byref(shape), 1, ctypes.byref(r), None, None, None,
                                ctypes.byref(st), 0.0, ctypes.byref(r), None, 256, 1 << 40,
                                None) == ck.EINVAL


def test_store_calls_refuse(lib):
    st, r = store(), rows()
    assert lib.certkv_store_workspace_bytes(0) == 0
    need = lib.certkv_store_workspace_bytes(16)
    assert need >= 4 * 17

    def load(packed=None, tail=1, reserve=0, ws=256, n=need, **kw):
        f = dict(k=FAKE, v=FAKE, offsets=FAKE, real_counts=FAKE, positions=None, capacity_slots=9)
        f.update(kw)
        p = ck.certkv_packed(*f.values())
        return lib.certkv_store_load(ctypes.byref(p), tail, reserve, ctypes.byref(st), ws, n, None)

    for kw in (dict(k=None), dict(v=FAKE + 8), dict(offsets=None), dict(offsets=FAKE + 4),
               dict(real_counts=None), dict(capacity_slots=0), dict(tail=2), dict(reserve=-1)):
        assert load(**kw) == ck.EINVAL, kw
    for kw in (dict(ws=None), dict(ws=128), dict(n=need - 1)):
        assert load(**kw) == ck.EWORKSPACE, kw

    def append(b=2, l=4, h=2, t=3, k=r, v=r, sel=None, acc=None, start=None):
        ref = [ctypes.byref(x) if x is not None else None for x in (k, v)]
        return lib.certkv_store_append(b, l, h, t, *ref, sel, acc, start, ctypes.byref(st), None)

    for kw in (dict(b=0), dict(l=3), dict(h=0), dict(t=0), dict(t=(1 << 24) + 1), dict(k=None),
               dict(v=rows(FAKE + 2)), dict(k=rows(st=4)), dict(sel=FAKE + 1), dict(acc=FAKE + 2),
               dict(start=FAKE + 3)):
        assert append(**kw) == ck.EINVAL, kw

    def read(t=1, start=None, k=FAKE, v=FAKE):
        return lib.certkv_store_read(ctypes.byref(st), start, t, k, v, None)

    for kw in (dict(t=0), dict(start=FAKE + 2), dict(k=None), dict(v=FAKE + 8)):
        assert read(**kw) == ck.EINVAL, kw


def test_tree_attn_refuses(lib):
    def shape(**kw):
        f = dict(batch=2, layers=4, hq=8, hkv=2, n=2, d=128, w=1)
        f.update(kw)
        return ck.certkv_shape(*f.values())

    good = shape()
    need = lib.certkv_tree_workspace_bytes(ctypes.byref(good), 8)
    assert need > 0
    for bad, t in ((shape(d=64), 8), (shape(batch=0), 8), (shape(hq=7), 8), (shape(hq=66), 8),
                   (good, 0), (good, 65)):
        assert lib.certkv_tree_workspace_bytes(ctypes.byref(bad), t) == 0

    def call(sh=good, t=8, q=rows(), k=None, v=None, mask=None, st=store(), scale=0.0, out=rows(),
             lse=None, ws=256, n=need):
        ref = [ctypes.byref(x) if x is not None else None for x in (q, k, v)]
        return lib.certkv_tree_attn(ctypes.byref(sh) if sh else None, t, *ref, mask,
                                    ctypes.byref(st) if st else None, scale,
                                    ctypes.byref(out) if out is not None else None, lse, ws, n,
                                    None)

    for kw in (dict(sh=None), dict(sh=shape(d=64)), dict(sh=shape(hq=66)), dict(t=0), dict(t=65),
               dict(q=None), dict(q=rows(FAKE + 2)), dict(q=rows(sh=100)), dict(k=rows()),
               dict(v=rows()), dict(k=rows(), v=rows(st=12)), dict(mask=FAKE + 4), dict(st=None),
               dict(st=store(units=15)), dict(scale=-1.0), dict(scale=float("nan")),
               dict(out=None), dict(out=rows(st=0)), dict(out=rows(sh=8)), dict(lse=FAKE + 2)):
        assert call(**kw) == ck.EINVAL, kw
    for kw in (dict(ws=None), dict(ws=64), dict(n=need - 1)):
        assert call(**kw) == ck.EWORKSPACE, kw


def test_binding_refuses_wrong_tensors():
    t = torch.zeros((1, 1, 2, 4, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        ck._rows(t, "q")
    with pytest.raises(TypeError):
        ck._rows(t.float(), "q")
    with pytest.raises(TypeError):
        ck._rows(t[..., :64], "q")
    with pytest.raises(ValueError):
        ck._index(torch.zeros(3, dtype=torch.int64), "accepted", (3,))
    with pytest.raises(ValueError):
        ck.Store(k=torch.zeros((2, 64, 64)), v=torch.zeros((2, 64, 64)),
                 table=torch.zeros((1, 2), dtype=torch.int32),
                 counts=torch.zeros(1, dtype=torch.int32), format="fp8")
    with pytest.raises(ValueError):
        ck.Store(k=torch.zeros((2, 64, 128), dtype=torch.uint8),
                 v=torch.zeros((2, 64, 128), dtype=torch.uint8),
                 table=torch.zeros((1, 2), dtype=torch.int32),
                 counts=torch.zeros(1, dtype=torch.int32), format="fp8")
