"""Refusals of the gradients of tree attention: every argument is checked on the host before
anything is launched (CPU only; no call reaches a GPU)."""
import ctypes

import pytest

from paper_2608_21541_gb300 import build as B
from paper_2608_21541_gb300 import certkv as ck
from test_drafts_abi import BAD_STORES, FAKE, store


@pytest.fixture(scope="module")
def lib():
    B.build()
    return ck.load_library()


def rows(data=FAKE, sb=1 << 20, sl=1 << 18, st=4096, sh=128):
    return ck.certkv_rows(data, sb, sl, st, sh)


def shape(**kw):
    s = dict(batch=2, layers=2, hq=16, hkv=4, n=2, d=128, w=1)
    s.update(kw)
    return ck.certkv_shape(**s)


BAD_SHAPES = [dict(batch=0), dict(layers=0), dict(hq=0), dict(hkv=0), dict(d=64), dict(hq=18),
              dict(hq=4 * 33), dict(batch=1 << 20, layers=32)]


def test_workspace(lib):
    def size(T=8, **kw):
        return lib.certkv_tree_grad_workspace_bytes(ctypes.byref(shape(**kw)), T)

    assert size() > 0 and size(T=64) > size()
    for kw in BAD_SHAPES + [dict(T=0), dict(T=65), dict(T=-1)]:
        assert size(**kw) == 0, kw
    assert lib.certkv_tree_grad_workspace_bytes(None, 8) == 0


def test_grad_refuses(lib):
    need = lib.certkv_tree_grad_workspace_bytes(ctypes.byref(shape()), 8)

    def call(sh=shape(), T=8, q=rows(), kn=rows(), vn=rows(), mask=FAKE, st=store(), scale=0.0,
             out=rows(), lse=FAKE, dout=rows(), dlse=FAKE, dq=rows(), dk=rows(), dv=rows(), ks=FAKE,
             vs=FAKE, ws=FAKE, n=need):
        ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return lib.certkv_tree_attn_grad(ref(sh), T, ref(q), ref(kn), ref(vn), mask, ref(st), scale,
                                         ref(out), lse, ref(dout), dlse, ref(dq), ref(dk), ref(dv),
                                         ks, vs, ws, n, None)

    for kw in BAD_SHAPES:
        assert call(sh=shape(**kw)) == ck.EINVAL, kw
    for kw in BAD_STORES + [dict(units=8)]:
        assert call(st=store(**kw)) == ck.EINVAL, kw
    off, gap = rows(data=FAKE + 8), rows(st=1028)
    overlap = rows(sb=1 << 18, sl=1 << 16, st=64)
    for kw in (dict(sh=None), dict(st=None), dict(T=0), dict(T=65), dict(q=None), dict(out=None),
               dict(dout=None), dict(q=off), dict(out=gap), dict(dout=off), dict(lse=None),
               dict(lse=FAKE + 2), dict(dlse=FAKE + 1), dict(mask=FAKE + 4), dict(kn=None),
               dict(vn=None), dict(kn=off), dict(vn=gap), dict(dq=off), dict(dq=overlap),
               dict(dq=rows(st=0)), dict(dk=None), dict(dv=None), dict(dk=overlap), dict(dv=gap),
               dict(kn=None, vn=None), dict(ks=None), dict(vs=None), dict(ks=FAKE + 64),
               dict(vs=FAKE + 16), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(dq=None, dk=None, dv=None, ks=None, vs=None),
               dict(kn=None, vn=None, dk=None, dv=None, dq=None, ks=None, vs=None)):
        assert call(**kw) == ck.EINVAL, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(n=need - 1), dict(n=0)):
        assert call(**kw) == ck.EWORKSPACE, kw
