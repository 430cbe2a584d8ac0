"""Rows that take no part in the gradients (their log-sum-exp is -inf: padding of a batch, or rows that
saw nothing) over segments with stored slots that hold NaN or infinities: they get 0 and give nothing."""
import pytest
import torch

import drafts
from test_gpu_grad import FORMATS, grads, step
from test_gpu_tree import store_with

pytestmark = pytest.mark.gpu

SHAPES = [(1, 4), (4, 2), (16, 4), (33, 4), (64, 8)]  # one pass for all gradients, and one each


def spoil(st, u, slot, value, name):
    """Slot `slot` of segment u holds `value`, as its row would that is appended with it."""
    at = int(drafts.slots(st.table.cpu().numpy(), u, slot, 1)[0])
    if st.format == "bf16":
        getattr(st, name).view(-1, 128)[at, 5] = value
        return at
    # a quantised row with a NaN or infinity is held as zeros with scale NaN
    getattr(st, name).view(torch.uint8).view(st.k.shape[0] * 64, -1)[at] = 0
    if st.format == "fp4":
        getattr(st, name + "_group").view(torch.uint8).view(-1, 8)[at] = 0
    getattr(st, name + "_scale").view(-1)[at] = float("nan")
    return at


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", SHAPES)
@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("name,value", [("k", float("nan")), ("k", float("inf")), ("v", float("nan")),
                                        ("v", -float("inf"))])
def test_padding_over_slots_that_are_not_finite(fmt, T, G, new, name, value):
    """Sequence 1 is padding throughout, sequence 0's last query head of its last token too."""
    H, counts = 2, [200, 70]
    st, n = store_with(counts, 2, 1, H, fmt, 400)
    x = step(st, 2, 1, H, G, T, new=new, seed=T)
    x["lse"][1] = -float("inf")
    x["lse"][0, :, -1, -1] = -float("inf")
    want = grads(st, x, H)  # over a store that is clean
    bad = [spoil(st, u, s, value, name) for u in range(4) for s in (3, 66)]
    for pools in (True, False):
        got = grads(st, x, H, pools=pools)
        assert not got["dq"][1].float().any(), "padding got a gradient"
        assert not got["dq"][0, :, -1, -1].float().any()
        if new:
            for d in ("dk", "dv"):
                assert not got[d][1].float().any()
                assert torch.equal(got[d], want[d])
        if not pools:
            continue
        table = st.table.cpu().numpy()
        for d in ("dk_store", "dv_store"):
            rows = got[d].view(-1, 128)
            for u in (2, 3):  # padding gave nothing, not even to the slots that are not finite
                assert not rows[torch.from_numpy(drafts.slots(table, u, 0, n[u])).cuda()].float().any(), (d, u)
            clean = torch.ones(len(rows), dtype=torch.bool, device="cuda")
            clean[bad] = False
            assert torch.equal(rows[clean], want[d].view(-1, 128)[clean]), d
        if name == "v" or value != value or fmt != "bf16":  # what does take part sees them
            assert torch.isnan(got["dk_store"].view(-1, 128)[bad[:4]].float()).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", SHAPES)
def test_padding_of_a_long_segment(fmt, T, G):
    """Segments that many blocks share, one head's rows all padding."""
    st, n = store_with([20000], 1, 1, 2, fmt, 410)
    x = step(st, 1, 1, 2, G, T, new=T % 2 == 0)
    x["lse"][:, :, :, :G] = -float("inf")
    at = int(drafts.slots(st.table.cpu().numpy(), 0, 12345, 1)[0])
    if fmt == "bf16":
        st.k.view(-1, 128)[at, 7] = float("nan")
    else:
        st.k_scale.view(-1)[at] = float("nan")
    got = grads(st, x, 2)
    assert not got["dq"][:, :, :, :G].float().any()
    assert torch.isfinite(got["dq"].float()).all() and got["dq"][:, :, :, G:].float().any()
    mine = torch.from_numpy(drafts.slots(st.table.cpu().numpy(), 0, 0, n[0])).cuda()
    for d in ("dk_store", "dv_store"):
        assert not got[d].view(-1, 128)[mine].float().any()
