"""Attention of a tree of drafted tokens over the paged store, against the definition in
64 bits on the values the store holds (tests/drafts.py states the bound)."""
import numpy as np
import pytest
import torch

import drafts
from drafts import PAGE, attention, check_attention, randn
from paper_2608_21541_gb300 import certkv as ck

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "fp8", "fp4")


def store_with(counts, B, L, H, fmt, seed, room=1, gain=1.0):
    """A store whose pages lie in no order and whose unused slots hold NaN patterns."""
    U = B * L * H
    counts = [counts[u % len(counts)] for u in range(U)]
    mp = max(1, -(-max(counts) // PAGE) + room)
    st = ck.Store.empty(U, mp, fmt)
    g = torch.Generator().manual_seed(seed)
    st.table.copy_(torch.randperm(U * mp, generator=g).view(U, mp))
    for name in ("k", "v"):
        getattr(st, name).view(torch.uint8).fill_(255)
        if fmt != "bf16":
            getattr(st, name + "_scale").fill_(float("nan"))
        if fmt == "fp4":
            getattr(st, name + "_group").view(torch.uint8).fill_(127)
    n = max(max(counts), 1)
    k, v = randn((B, L, n, H, 128), seed + 1, gain=gain), randn((B, L, n, H, 128), seed + 2)
    ck.certkv_store_append(k, v, st, start=torch.zeros(U, dtype=torch.int32).cuda())
    st.counts.copy_(torch.tensor(counts, dtype=torch.int32))
    # the slots past the live ones hold NaN again
    table = st.table.cpu().numpy()
    for u in range(U):
        at = torch.from_numpy(drafts.slots(table, u, counts[u], mp * PAGE - counts[u])).cuda()
        for name in ("k", "v"):
            getattr(st, name).view(torch.uint8).view(U * mp * PAGE, -1)[at] = 255
            if fmt != "bf16":
                getattr(st, name + "_scale").view(-1)[at] = float("nan")
    return st, counts


def words(B, T, seed):
    rng = np.random.default_rng(seed)
    return torch.tensor([drafts.random_tree(T, rng) for _ in range(B)], dtype=torch.int64).cuda()


def run(st, counts, B, L, H, G, T, mask=None, new=True, seed=0, gain=1.0, scale=0.0):
    q = randn((B, L, T, H * G, 128), seed + 3, gain=gain)
    k, v = (randn((B, L, T, H, 128), seed + 4 + i) if new else None for i in range(2))
    lse = torch.empty((B, L, T, H * G), device="cuda")
    out = ck.certkv_tree_attn(q, st, hkv=H, k_new=k, v_new=v, mask=mask, lse=lse, scale=scale)
    ref = attention(q, st, counts, H, k, v, mask, scale if scale else None)
    check_attention(out, lse, ref)
    return q, k, v, out, lse


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 8), (1, 32), (2, 3), (5, 8), (7, 16), (16, 4),
                                 (33, 2), (64, 1), (64, 5)])
def test_lengths_and_groups(fmt, T, G):
    B, L, H = 2, 1, 2
    counts = [0, 1, 63, 64, 65, 129, 500, 777]
    for i in range(0, len(counts), 4):
        st, n = store_with(counts[i:i + 4], B, L, H, fmt, 100 + i)
        run(st, n, B, L, H, G, T, mask=words(B, T, T + i), seed=i)
        assert st.read_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_chain_without_mask_and_without_new_keys(fmt):
    st, n = store_with([130, 7], 1, 2, 2, fmt, 200)
    run(st, n, 1, 2, 2, 4, 6)
    run(st, n, 1, 2, 2, 4, 6, new=False)
    run(st, n, 1, 2, 2, 4, 6, scale=0.5)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(3, 2), (40, 4), (64, 16)])
def test_rows_that_see_nothing(fmt, T, G):
    """An empty segment and a mask word of 0: output 0, log-sum-exp -inf; bits past
    the drafts are not looked at."""
    st, n = store_with([0, 90], 1, 1, 2, fmt, 210)
    mask = words(1, T, 5)
    mask[0, 1] = 0
    if T < 64:
        mask |= -1 << T  # bits past the drafts
    _, _, _, out, lse = run(st, n, 1, 1, 2, G, T, mask=mask)
    assert not out[0, 0, 1, :G].float().any() and torch.isinf(lse[0, 0, 1, :G]).all()
    out = ck.certkv_tree_attn(randn((1, 1, T, 2 * G, 128), 1), st, hkv=2)
    assert not out[0, 0, :, :G].float().any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(4, 2), (32, 4), (64, 8)])
def test_unseen_drafts_do_not_touch_a_row(fmt, T, G):
    """Drafts that hold NaN and infinities: rows that do not see them are bit for bit
    what they are without, rows that do are not finite."""
    st, n = store_with([200, 3], 1, 1, 2, fmt, 220)
    q = randn((1, 1, T, 2 * G, 128), 1)
    k, v = randn((1, 1, T, 2, 128), 2), randn((1, 1, T, 2, 128), 3)
    words = [(1 << t) | 1 if t % 2 else 1 for t in range(T)]
    mask = torch.tensor([[w - (1 << 64) if w >> 63 else w for w in words]]).cuda()
    mask[0, 2] = 1 | 1 << 2
    want = ck.certkv_tree_attn(q, st, hkv=2, k_new=k, v_new=v, mask=mask)
    k2, v2 = k.clone(), v.clone()
    v2[0, 0, 2, :, 9] = float("nan")
    v2[0, 0, 2, :, 10] = float("inf")
    if T > 5:  # token 4 is seen by nobody
        k2[0, 0, 4] = float("nan")
        v2[0, 0, 4] = float("-inf")
    got = ck.certkv_tree_attn(q, st, hkv=2, k_new=k2, v_new=v2, mask=mask)
    rest = [t for t in range(T) if t != 2]
    assert torch.equal(got[:, :, rest], want[:, :, rest])
    assert not torch.isfinite(got[0, 0, 2, :, 9:11].float()).any()
    keep = [d for d in range(128) if d not in (9, 10)]
    assert torch.equal(got[0, 0, 2][:, keep], want[0, 0, 2][:, keep])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 8), (64, 4)])
def test_values_of_very_different_size_and_large_logits(fmt, T, G):
    """Sharp rows (logits of hundreds) and value rows from 2^-12 to 2^12."""
    B, L, H, n = 1, 1, 2, 300
    st = ck.Store.empty(H, 6, fmt)
    g = torch.Generator().manual_seed(1)
    k, v = randn((B, L, n, H, 128), 70, gain=6.0), randn((B, L, n, H, 128), 71)
    v *= torch.exp2(torch.randint(-12, 13, (1, 1, n, 1, 1), generator=g).float()).cuda().bfloat16()
    ck.certkv_store_append(k, v, st)
    q = randn((B, L, T, H * G, 128), 72, gain=6.0)
    lse = torch.empty((B, L, T, H * G), device="cuda")
    out = ck.certkv_tree_attn(q, st, hkv=H, lse=lse)
    check_attention(out, lse, attention(q, st, [n] * H, H))


@pytest.mark.parametrize("fmt", ("fp8", "fp4"))
def test_small_values_behind_a_large_one(fmt):
    """A row whose weight lies on slots with small values, beside slots of large values
    that it hardly sees, keeps the small values' own accuracy."""
    st = ck.Store.empty(1, 2, fmt)
    k, v = randn((1, 1, 100, 1, 128), 73, gain=0.0), randn((1, 1, 100, 1, 128), 74)
    k[..., 0] = 0.0
    v[0, 0, 50] *= 4096.0
    k[0, 0, 50, 0, 0] = -64.0
    q = torch.zeros((1, 1, 1, 4, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 8.0  # logit -45 on slot 50
    ck.certkv_store_append(k, v, st)
    out = ck.certkv_tree_attn(q, st, hkv=1).double().cpu().numpy()
    ref, _, _, _ = attention(q, st, [100], 1)
    # the other slots' values are at most ~4: weights held to 2^-9 of those
    assert np.abs(out - ref).max() <= 2.0 ** -8 * 4.0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(3, 4), (40, 4)])
def test_missing_pages_are_left_out(fmt, T, G):
    st, n = store_with([300], 1, 1, 2, fmt, 230)
    st.table[0, 1] = -1
    st.table[1, 0] = st.k.shape[0]
    st.table[1, 4] = -7
    at = st.table.clone()
    at[1, 0] = -1  # what the definition calls no page
    q = randn((1, 1, T, 2 * G, 128), 1)
    out = ck.certkv_tree_attn(q, st, hkv=2)
    assert st.read_status() == ck.STATUS_STORE
    ref = ck.Store(k=st.k, v=st.v, table=at, counts=st.counts, format=fmt, k_group=st.k_group,
                   v_group=st.v_group, k_scale=st.k_scale, v_scale=st.v_scale)
    check_attention(out, None, attention(q, ref, n, 2))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 4), (24, 4), (64, 8)])
def test_a_row_that_is_not_finite_stays_alone(fmt, T, G):
    """A query row with a NaN makes its own output NaN and nothing else's."""
    st, n = store_with([400, 70], 1, 1, 2, fmt, 240)
    q = randn((1, 1, T, 2 * G, 128), 1)
    k, v = randn((1, 1, T, 2, 128), 2), randn((1, 1, T, 2, 128), 3)
    want = ck.certkv_tree_attn(q, st, hkv=2, k_new=k, v_new=v)
    q[0, 0, T - 1, 1, 7] = float("nan")
    got = ck.certkv_tree_attn(q, st, hkv=2, k_new=k, v_new=v)
    assert torch.isnan(got[0, 0, T - 1, 1].float()).all()
    got[0, 0, T - 1, 1] = want[0, 0, T - 1, 1]
    assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", (1, 12, 48))
def test_views_streams_graphs_and_repeats(fmt, T):
    """Views of a fused projection and a transposed output give the bits of dense
    tensors; so do another stream, a replayed graph and ten repeats."""
    B, L, H, G = 2, 2, 2, 4
    st, n = store_with([700, 64, 0, 333], B, L, H, fmt, 250)
    x = randn((B, L, T, H * (G + 2), 128), 9)
    q, k, v = x[..., :H * G, :], x[..., H * G:H * (G + 1), :], x[..., H * (G + 1):, :]
    mask = words(B, T, 3)
    want = ck.certkv_tree_attn(q.contiguous(), st, hkv=H, k_new=k.contiguous(),
                               v_new=v.contiguous(), mask=mask)
    out = torch.empty((B, H * G, T, L, 128), dtype=torch.bfloat16, device="cuda").permute(0, 3, 2, 1, 4)
    ck.certkv_tree_attn(q, st, hkv=H, k_new=k, v_new=v, mask=mask, out=out)
    assert torch.equal(out, want)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = ck.certkv_tree_attn(q, st, hkv=H, k_new=k, v_new=v, mask=mask, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    ws = ck.workspace(ck.certkv_tree_workspace_bytes(B, L, H * G, H, T), "cuda")
    for _ in range(10):  # a workspace that holds anything
        ws.random_()
        got = ck.certkv_tree_attn(q, st, hkv=H, k_new=k, v_new=v, mask=mask, ws=ws)
        assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    out = torch.zeros_like(want)
    with torch.cuda.graph(g):
        ck.certkv_tree_attn(q, st, hkv=H, k_new=k, v_new=v, mask=mask, out=out, ws=ws)
    st.counts[0] = 123  # a replay reads the current counts
    g.replay()
    torch.cuda.synchronize()
    n[0] = 123
    check_attention(out, None, attention(q, st, n, H, k, v, mask))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G,n", [(1, 4, 20011), (3, 8, 9001), (16, 4, 20011), (64, 4, 4099)])
def test_long_segments_are_split_and_joined(fmt, T, G, n):
    st, c = store_with([n], 1, 1, 1, fmt, 260)
    run(st, c, 1, 1, 1, G, T, mask=words(1, T, 1), gain=2.0)


def test_matches_decode_over_the_packed_cache():
    """A bf16 store loaded from a compressed cache: one token without keys of its own
    is the framework's own decode."""
    from paper_2608_21541_gb300 import workloads as W
    wl = W.WORKLOADS["C1"].with_(n=4096, w=16)
    K, V, Q = W.draw(wl, device="cuda")
    packed = ck.certkv_compress(K, V, Q, wl.B_live)
    st = ck.Store.empty(wl.H, 65, "bf16", pool_pages=200)
    ck.certkv_store_load(packed, st)
    q = W.draw_decode_queries(wl, 0, device="cuda")
    a = ck.certkv_decode_attn(q, packed, hkv=wl.H).float()
    b = ck.certkv_tree_attn(q.unsqueeze(2), st, hkv=wl.H)[:, :, 0].float()
    assert (a - b).abs().max() <= 2.0 ** -7 * a.abs().max()


@pytest.mark.parametrize("T,G", [(1, 4), (9, 8)])
@pytest.mark.parametrize("units", [255, 256, 257, 1100])
def test_many_segments(units, T, G):
    """Around the number of segments up to which a CTA scans the lengths itself, and
    more than one block's scan takes in one go."""
    st, n = store_with([3, 0, 70, 129, 1], 1, units, 1, "fp8", 270)
    q = randn((1, units, T, G, 128), 1)
    k, v = randn((1, units, T, 1, 128), 2), randn((1, units, T, 1, 128), 3)
    out = ck.certkv_tree_attn(q, st, hkv=1, k_new=k, v_new=v)
    check_attention(out, None, attention(q, st, n, 1, k, v))
    alone = ck.Store(k=st.k, v=st.v, table=st.table[-2:], counts=st.counts[-2:], format="fp8",
                     k_scale=st.k_scale, v_scale=st.v_scale)
    two = ck.certkv_tree_attn(q[:, -2:], alone, hkv=1, k_new=k[:, -2:], v_new=v[:, -2:])
    # the same rows, split over the CTAs in another way
    assert (two.float() - out[:, -2:].float()).abs().max() <= 2.0 ** -7 * out.float().abs().max()


def test_no_slots_anywhere():
    st, _ = store_with([0], 2, 1, 3, "bf16", 280)
    q = randn((2, 1, 4, 6, 128), 1)
    lse = torch.empty((2, 1, 4, 6), device="cuda")
    out = ck.certkv_tree_attn(q, st, hkv=3, lse=lse)
    assert not out.float().any() and torch.isinf(lse).all() and (lse < 0).all()


@pytest.mark.parametrize("fmt,pages", [("bf16", 262144 + 9), ("fp8", 524288 + 9), ("fp4", 1048576 + 9)])
@pytest.mark.parametrize("T,G", [(1, 4), (9, 16)])
def test_pool_past_thirty_two_bits_of_bytes(fmt, pages, T, G):
    """Pages at the end of a pool whose codes pass 2^32 bytes."""
    small, n = store_with([300, 65], 1, 1, 2, fmt, 290)
    st = ck.Store.empty(2, small.table.shape[1], fmt, pool_pages=pages)
    old = [p for p in small.table.flatten().tolist() if p >= 0]
    new = [pages - 1 - i for i in range(len(old))]
    for name in ("k", "v", "k_scale", "v_scale", "k_group", "v_group"):
        a, b = getattr(small, name), getattr(st, name)
        if a is not None:
            b.view(torch.uint8)[new] = a.view(torch.uint8)[old]
    move = dict(zip(old, new))
    st.table.copy_(torch.tensor([[move.get(p, -1) for p in row] for row in small.table.tolist()]))
    st.counts.copy_(small.counts)
    q = randn((1, 1, T, 2 * G, 128), 1)
    kw = dict(hkv=2)
    assert torch.equal(ck.certkv_tree_attn(q, st, **kw), ck.certkv_tree_attn(q, small, **kw))
