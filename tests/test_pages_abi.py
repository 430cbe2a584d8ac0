"""Refusals of the operators that keep a store's pages: every argument is checked on the host
before anything is launched (CPU only; no call reaches a GPU)."""
import ctypes

import pytest
import torch

from paper_2608_21541_gb300 import build as B
from paper_2608_21541_gb300 import certkv as ck
from test_drafts_abi import BAD_STORES, FAKE, store


@pytest.fixture(scope="module")
def lib():
    B.build()
    return ck.load_library()


BAD_PAGES = [dict(held=None), dict(free=None), dict(free_count=None), dict(held=FAKE + 2),
             dict(free=FAKE + 1), dict(free_count=FAKE + 3)]


def pages(**kw):
    f = dict(held=FAKE, free=FAKE, free_count=FAKE)
    f.update(kw)
    return ck.certkv_pages(*f.values())


def test_workspace(lib):
    size = lib.certkv_pages_workspace_bytes
    assert size(16, 64) % 256 == 0 and size(16, 64) > 0
    assert size(1 << 24, (1 << 25) - 1) > size(16, 64)
    for units, pool in ((0, 64), (-1, 64), ((1 << 24) + 1, 64), (16, 0), (16, 1 << 25)):
        assert size(units, pool) == 0


def test_list_refuses(lib):
    need = lib.certkv_pages_workspace_bytes(16, 64)

    def call(st=store(), pg=pages(), ws=FAKE, n=need):
        return lib.certkv_pages_list(ctypes.byref(st) if st else None,
                                     ctypes.byref(pg) if pg else None, ws, n, None)

    for kw in BAD_STORES:
        assert call(st=store(**kw)) == ck.EINVAL, kw
    for kw in BAD_PAGES:
        assert call(pg=pages(**kw)) == ck.EINVAL, kw
    assert call(st=None) == ck.EINVAL and call(pg=None) == ck.EINVAL
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(n=need - 1), dict(n=0)):
        assert call(**kw) == ck.EWORKSPACE, kw


def test_reserve_refuses(lib):
    need = lib.certkv_pages_workspace_bytes(16, 64)

    def call(batch=2, room=FAKE, want=FAKE, st=store(), pg=pages(), ws=FAKE, n=need):
        return lib.certkv_pages_reserve(batch, room, want, ctypes.byref(st) if st else None,
                                        ctypes.byref(pg) if pg else None, ws, n, None)

    for kw in BAD_STORES:
        assert call(st=store(**kw)) == ck.EINVAL, kw
    for kw in BAD_PAGES:
        assert call(pg=pages(**kw)) == ck.EINVAL, kw
    for kw in (dict(batch=0), dict(batch=-2), dict(batch=3), dict(batch=32), dict(room=FAKE + 1),
               dict(want=FAKE + 2), dict(st=None), dict(pg=None)):
        assert call(**kw) == ck.EINVAL, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 64), dict(n=need - 1)):
        assert call(**kw) == ck.EWORKSPACE, kw


def test_slot_map_refuses(lib):
    def call(batch=2, tokens=8, rows=FAKE, start=FAKE, base=FAKE, mask=FAKE, st=store(), slots=FAKE,
             pos=FAKE):
        return lib.certkv_slot_map(batch, tokens, rows, start, base, mask,
                                   ctypes.byref(st) if st else None, slots, pos, None)

    for kw in BAD_STORES:
        assert call(st=store(**kw)) == ck.EINVAL, kw
    for kw in (dict(batch=0), dict(batch=3), dict(tokens=0), dict(tokens=65), dict(rows=FAKE + 1),
               dict(start=FAKE + 2), dict(base=FAKE + 3), dict(mask=FAKE + 4), dict(slots=FAKE + 1),
               dict(pos=FAKE + 2), dict(slots=None, pos=None), dict(st=None),
               dict(tokens=1 << 30, mask=None, st=store(units=1 << 20))):
        assert call(**kw) == ck.EINVAL, kw


@pytest.mark.parametrize("tokens", [2 ** 30 + 1, 2 ** 31 - 1])
def test_slot_map_refuses_rows_past_its_counting(lib, tokens):
    """Rows are counted in 32 bits, a block's worth past the last."""
    st = store()
    assert lib.certkv_slot_map(2, tokens, None, None, None, None, ctypes.byref(st), FAKE, None,
                               None) == ck.EINVAL


def test_binding_refuses():
    with pytest.raises(ValueError):
        ck.Pages(held=torch.zeros(4, dtype=torch.int64), free=torch.zeros(4, dtype=torch.int32),
                 free_count=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        ck.Pages(held=torch.zeros(4, dtype=torch.int32), free=torch.zeros(4, dtype=torch.int32),
                 free_count=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):  # not on a GPU
        ck.Pages(held=torch.zeros(4, dtype=torch.int32), free=torch.zeros(4, dtype=torch.int32),
                 free_count=torch.zeros(1, dtype=torch.int32))
