"""The paged store against its definition: codes, scales, pages and counts equal bit
for bit what the fp32 steps of the definition give; reading back is one bf16
rounding of the values held."""
import numpy as np
import pytest
import torch

import drafts
from drafts import PAGE, encode, held, slots, values
from paper_2608_21541_gb300 import certkv as ck

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp8", "fp4")


def same(got, at, enc):
    np.testing.assert_array_equal(got["codes"][at], enc["codes"])
    np.testing.assert_array_equal(got["scale"][at], enc["scale"])
    if "group" in enc:
        np.testing.assert_array_equal(got["group"][at], enc["group"])


def odd_rows(n, seed):
    """Rows of many magnitudes: zeros, subnormal and huge rows, one element alone,
    equal elements, rounding ties."""
    x = drafts.randn((n, 128), seed).float().cpu()
    g = torch.Generator().manual_seed(seed + 1)
    x *= torch.exp2(torch.randint(-20, 20, (n, 1), generator=g).float())
    if n > 8:
        x[0] = 0
        x[1] = 0
        x[1, 77] = -3.0
        x[2] *= 2.0 ** -110  # flushed
        x[3] = 1e-39
        x[4] *= 2.0 ** 100
        x[5] = 1.75
        x[6] = torch.arange(128) * 0.25
        x[7, 16:32] = 0
        x[8, :64] *= 2.0 ** -30
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts,tail,reserve", [([1, 64, 65, 200, 3], 1, 0),
                                                 ([0, 5, 127, 1], 0, 1), ([1], 1, 64)])
def test_load_packed(fmt, counts, tail, reserve):
    n = np.array(counts) + tail
    off = np.concatenate([[0], np.cumsum(n)])
    rows = [odd_rows(int(off[-1]), 10 + i) for i in range(2)]
    packed = ck.Packed(k=rows[0].cuda(), v=rows[1].cuda(), offsets=torch.tensor(off).cuda(),
                       real_counts=torch.tensor(counts, dtype=torch.int32).cuda(),
                       positions=torch.zeros(int(off[-1]), dtype=torch.int32).cuda(),
                       tail_slot=tail)
    pages = -(-(n + reserve) // PAGE)
    mp = int(pages.max()) + 1
    st = ck.Store.empty(len(n), mp, fmt, pool_pages=int(pages.sum()) + 2)
    ck.certkv_store_load(packed, st, reserve)
    assert st.read_status() == 0
    np.testing.assert_array_equal(st.counts.cpu().numpy(), n)
    first = np.cumsum(pages) - pages
    want = np.where(np.arange(mp) < pages[:, None], first[:, None] + np.arange(mp), -1)
    table = st.table.cpu().numpy()
    np.testing.assert_array_equal(table, want)
    at = np.concatenate([slots(table, u, 0, int(n[u])) for u in range(len(n))])
    for name, r in zip("kv", rows):
        same(held(st, name), at, encode(r, fmt))


@pytest.mark.parametrize("fmt", FORMATS)
def test_load_cuts_where_the_pool_ends(fmt):
    n = np.array([130, 200, 70])
    off = np.concatenate([[0], np.cumsum(n)])
    rows = drafts.randn((int(off[-1]), 128), 20)
    packed = ck.Packed(k=rows, v=rows, offsets=torch.tensor(off).cuda(),
                       real_counts=torch.tensor(n, dtype=torch.int32).cuda(),
                       positions=torch.zeros(400, dtype=torch.int32).cuda(), tail_slot=0)
    st = ck.Store.empty(3, 3, fmt, pool_pages=5)  # wants 3 + 4 + 2 pages, rows of 3
    ck.certkv_store_load(packed, st)
    assert st.read_status() == ck.STATUS_STORE
    np.testing.assert_array_equal(st.counts.cpu().numpy(), [130, 128, 0])
    np.testing.assert_array_equal(st.table.cpu().numpy(), [[0, 1, 2], [3, 4, -1], [-1, -1, -1]])
    same(held(st, "k"), slots(st.table.cpu().numpy(), 1, 0, 128),
         encode(rows[130:258].cpu(), fmt))
    # a segment that does not lie in the packed cache is left out
    packed.offsets[2] = 1 << 40
    st2 = ck.Store.empty(3, 4, fmt, pool_pages=12)
    ck.certkv_store_load(packed, st2)
    assert st2.read_status() == ck.STATUS_STORE
    assert st2.counts.tolist() == [130, 200, 0]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,L,H,T,heads_first", [(1, 1, 1, 1, False), (2, 2, 3, 9, False),
                                                 (1, 2, 2, 150, True)])
def test_append_and_read_back(fmt, B, L, H, T, heads_first):
    U = B * L * H
    k, v = (odd_rows(U * T, 30 + i).view(B, L, H, T, 128).cuda() for i in range(2))
    rows = [x.reshape(U, T, 128).cpu() for x in (k, v)]
    if heads_first:
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    else:
        k, v = (x.transpose(2, 3).contiguous() for x in (k, v))
    mp = 5
    st = ck.Store.empty(U, mp, fmt)
    g = torch.Generator().manual_seed(5)
    st.table.copy_(torch.randperm(U * mp, generator=g).view(U, mp))
    start = torch.randint(0, 130, (U,), generator=g, dtype=torch.int32)
    ck.certkv_store_append(k, v, st, start=start.cuda())
    np.testing.assert_array_equal(st.counts.cpu().numpy(), start.numpy() + T)
    table = st.table.cpu().numpy()
    for name, r in zip("kv", rows):
        got = held(st, name)
        for u in range(U):
            same(got, slots(table, u, int(start[u]), T), encode(r[u], fmt))
    got = ck.certkv_store_read(st, T + 3, start=start.cuda())
    for x, r in zip(got, rows):
        x = x.cpu()
        assert not x[:, T:].float().any()
        for u in range(U):
            ref = torch.from_numpy(values(encode(r[u], fmt)))
            d = (x[u, :T].double() - ref).abs()
            # one rounding of code x scale to fp32 (two with a group scale) and one to bf16
            assert (d <= ref.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-40).all()
    # appended after the live slots: the same rows again, behind the first ones
    ck.certkv_store_append(k[:, :, :1], v[:, :, :1], st)
    np.testing.assert_array_equal(st.counts.cpu().numpy(), start.numpy() + T + 1)
    got = held(st, "k")
    for u in range(U):
        same(got, slots(table, u, int(start[u]) + T, 1), encode(rows[0][u, :1], fmt))
    assert st.read_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_the_accepted_path(fmt):
    B, L, H, T = 3, 2, 2, 8
    k, v = drafts.randn((B, L, T, H, 128), 40), drafts.randn((B, L, T, H, 128), 41)
    st = ck.Store.empty(B * L * H, 2, fmt)
    for name in "kv":
        getattr(st, name).view(torch.uint8).fill_(17)
    st.counts.fill_(61)
    accepted = torch.tensor([3, 0, 8], dtype=torch.int32).cuda()
    select = torch.tensor([[0, 2, 7, -9, 99, 0, 0, 0], [99] * 8, [0, 1, 2, 3, 4, 5, 6, 7]],
                          dtype=torch.int32).cuda()
    before = st.k.view(torch.uint8).clone()
    ck.certkv_store_append(k, v, st, select=select, accepted=accepted)
    assert st.read_status() == 0  # entries past the accepted ones are not looked at
    acc, sel = accepted.tolist(), select.tolist()
    table = st.table.cpu().numpy()
    got = {name: held(st, name) for name in "kv"}
    for u in range(B * L * H):
        b, l, h = u // (L * H), u // H % L, u % H
        assert st.counts[u].item() == 61 + acc[b]
        for name, x in (("k", k), ("v", v)):
            r = x[b, l, sel[b][:acc[b]], h].cpu()
            if acc[b]:
                same(got[name], slots(table, u, 61, acc[b]), encode(r, fmt))
        tail = slots(table, u, 61 + acc[b], 8)
        assert torch.equal(st.k.view(torch.uint8).view(-1, before.shape[-1])[tail],
                           before.view(-1, before.shape[-1])[tail])


def test_append_past_the_table_is_skipped_and_reported():
    st = ck.Store.empty(2, 2, "fp8")
    st.table[1, 1] = -1
    k = drafts.randn((1, 1, 10, 2, 128), 50)
    start = torch.tensor([120, 60], dtype=torch.int32).cuda()
    ck.certkv_store_append(k, k, st, start=start)
    assert st.read_status() == ck.STATUS_STORE
    assert st.counts.tolist() == [128, 70]
    got = held(st, "k")
    same(got, slots(st.table.cpu().numpy(), 0, 120, 8), encode(k[0, 0, :8, 0].cpu(), "fp8"))
    # slots without a page read as 0
    rows, _ = ck.certkv_store_read(st, 10, start=start)
    assert not rows[1, 4:].float().any() and rows[1, :4].float().abs().sum() > 0
    for bad in (dict(select=torch.full((1, 10), 10, dtype=torch.int32).cuda()),
                dict(accepted=torch.tensor([11], dtype=torch.int32).cuda())):
        st.status.zero_()
        st.counts.zero_()
        ck.certkv_store_append(k, k, st, **bad)
        assert st.read_status() == ck.STATUS_STORE
        assert st.counts.tolist() == [10, 10]


@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_rows_that_are_not_finite_read_as_nan(fmt):
    k = drafts.randn((1, 1, 4, 1, 128), 60)
    k[0, 0, 1, 0, 5] = float("nan")
    k[0, 0, 2, 0, 127] = float("-inf")
    st = ck.Store.empty(1, 1, fmt)
    ck.certkv_store_append(k, k, st)
    x = ck.certkv_store_read(st, 4)[0].float()[0]
    assert torch.isnan(x[1:3]).all() and torch.isfinite(x[[0, 3]]).all()


def test_read_outside_the_live_slots():
    st = ck.Store.empty(2, 2, "bf16")
    k = drafts.randn((1, 1, 70, 2, 128), 61)
    ck.certkv_store_append(k, k, st)
    x, _ = ck.certkv_store_read(st, 5, start=torch.tensor([-2, 68], dtype=torch.int32).cuda())
    assert not x[0, :2].float().any() and torch.equal(x[0, 2:], k[0, 0, :3, 0])
    assert torch.equal(x[1, :2], k[0, 0, 68:, 1]) and not x[1, 2:].float().any()


def test_pool_past_thirty_two_bits_of_bytes():
    """Pages whose byte offset passes 2^32, and whose element offset passes 2^31."""
    st = ck.Store.empty(1, 2, "bf16", pool_pages=300000)
    st.table[0] = torch.tensor([299999, 270001], dtype=torch.int32)
    k, v = drafts.randn((1, 1, 100, 1, 128), 62), drafts.randn((1, 1, 100, 1, 128), 63)
    ck.certkv_store_append(k, v, st)
    x, y = ck.certkv_store_read(st, 100)
    assert torch.equal(x[0], k[0, 0, :, 0]) and torch.equal(y[0], v[0, 0, :, 0])
    assert torch.equal(st.k[299999], k[0, 0, :64, 0])
    q = drafts.randn((1, 1, 2, 4, 128), 64)
    got = ck.certkv_tree_attn(q, st, hkv=1)
    small = ck.Store.empty(1, 2, "bf16")
    ck.certkv_store_append(k, v, small)
    assert torch.equal(got, ck.certkv_tree_attn(q, small, hkv=1))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", [127, 128, 129, 255, 256, 257, 401])
def test_append_many_rows(fmt, T):
    """Lengths around a block's rows; some accepted, chosen in reverse, one segment
    started before its first slot and one short of a page."""
    B, L, H = 2, 1, 3
    k, v = drafts.randn((B, L, T, H, 128), 70), drafts.randn((B, L, T, H, 128), 71)
    mp = 8
    st = ck.Store.empty(B * L * H, mp, fmt)
    for name in "kv":
        getattr(st, name).view(torch.uint8).fill_(17)
    st.table[1, 1] = -1
    accepted = [T, T - 60]
    select = torch.arange(T - 1, -1, -1, dtype=torch.int32).repeat(B, 1)
    starts = [3, 60, -2, 100, 0, mp * PAGE - 5]
    before = held(st, "k")
    ck.certkv_store_append(k, v, st, select=select.cuda(), start=torch.tensor(starts, dtype=torch.int32).cuda(),
                           accepted=torch.tensor(accepted, dtype=torch.int32).cuda())
    assert st.read_status() == ck.STATUS_STORE
    table = st.table.cpu().numpy()
    got = {name: held(st, name) for name in "kv"}
    written = set()
    for u in range(B * L * H):
        b, h, m = u // H, u % H, accepted[u // H]
        assert st.counts[u].item() == min(max(starts[u], 0) + m, mp * PAGE)
        on = [i for i in range(m) if starts[u] >= 0 and starts[u] + i < mp * PAGE
              and table[u, (starts[u] + i) // PAGE] >= 0]
        at = [int(table[u, (starts[u] + i) // PAGE]) * PAGE + (starts[u] + i) % PAGE for i in on]
        written |= set(at)
        if on:
            for name, x in (("k", k), ("v", v)):
                rows = x[b, 0, [T - 1 - i for i in on], h].cpu()
                same(got[name], np.array(at), encode(rows, fmt))
    rest = np.array(sorted(set(range(B * L * H * mp * PAGE)) - written))
    np.testing.assert_array_equal(got["k"]["codes"][rest], before["codes"][rest])
