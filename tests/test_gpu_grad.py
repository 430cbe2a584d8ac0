"""Gradients of tree attention over the paged store, against the definition in 64 bits on the
values the store holds (tests/treegrad.py states the bound), and against differences."""
import numpy as np
import pytest
import torch

import treegrad
from drafts import randn
from paper_2608_21541_gb300 import certkv as ck
from test_gpu_tree import FORMATS, store_with, words

pytestmark = pytest.mark.gpu
FILL = 7.0  # what the store's gradients hold where nothing is written


def step(st, B, L, H, G, T, mask=None, new=True, seed=0, gain=1.0, scale=0.0, with_dlse=False):
    """Inputs of a step, and what the forward pass leaves of it."""
    x = dict(q=randn((B, L, T, H * G, 128), seed + 3, gain=gain),
             dout=randn((B, L, T, H * G, 128), seed + 9), mask=mask, scale=scale)
    x["k_new"], x["v_new"] = (randn((B, L, T, H, 128), seed + 4 + i) if new else None
                              for i in range(2))
    x["lse"] = torch.empty((B, L, T, H * G), device="cuda")
    x["out"] = ck.certkv_tree_attn(x["q"], st, hkv=H, k_new=x["k_new"], v_new=x["v_new"], mask=mask,
                                   scale=scale, lse=x["lse"])
    x["dlse"] = randn((B, L, T, H * G), seed + 11).float() if with_dlse else None
    return x


def grads(st, x, H, pools=True, **kw):
    got = {}
    if pools:
        shape = (st.k.shape[0], 64, 128)
        got = {n: torch.full(shape, FILL, dtype=torch.bfloat16, device="cuda")
               for n in ("dk_store", "dv_store")}
    got["dq"], got["dk"], got["dv"] = ck.certkv_tree_attn_grad(
        x["dout"], x["q"], st, x["out"], x["lse"], hkv=H, k_new=x["k_new"], v_new=x["v_new"],
        mask=x["mask"], scale=x["scale"], dlse=x["dlse"], dk_store=got.get("dk_store"),
        dv_store=got.get("dv_store"), **kw)
    return got


def check(st, counts, x, H, got):
    ref = treegrad.gradients(x["q"], st, counts, H, x["out"], x["lse"], x["dout"], x["k_new"],
                             x["v_new"], x["mask"], x["scale"] if x["scale"] else None, x["dlse"])
    for name, t in got.items():
        if t is None:
            continue
        treegrad.check(t, ref, name)
        if name.endswith("_store"):  # slots that are not live are left alone
            rest = np.isnan(ref[name][0]).all(1)
            assert (t.view(-1, 128)[torch.from_numpy(rest).cuda()] == FILL).all()


def run(st, counts, B, L, H, G, T, pools=True, **kw):
    x = step(st, B, L, H, G, T, **kw)
    got = grads(st, x, H, pools)
    check(st, counts, x, H, got)
    return x, got


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 8), (1, 32), (2, 3), (5, 8), (7, 16), (16, 4),
                                 (33, 2), (64, 1), (64, 2), (43, 3), (64, 5)])
def test_lengths_and_groups(fmt, T, G):
    B, L, H = 2, 1, 2
    counts = [0, 1, 63, 64, 65, 129, 500, 777]
    for i in range(0, len(counts), 4):
        st, n = store_with(counts[i:i + 4], B, L, H, fmt, 100 + i)
        run(st, n, B, L, H, G, T, mask=words(B, T, T + i), seed=i)
        assert st.read_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_chain_no_new_keys_scale_dlse(fmt):
    st, n = store_with([130, 7], 1, 2, 2, fmt, 200)
    run(st, n, 1, 2, 2, 4, 6)
    run(st, n, 1, 2, 2, 4, 6, new=False)
    run(st, n, 1, 2, 2, 4, 6, scale=0.5)
    run(st, n, 1, 2, 2, 4, 6, with_dlse=True)
    run(st, n, 1, 2, 2, 4, 6, pools=False)
    run(st, n, 1, 2, 2, 16, 30, with_dlse=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_large_logits(fmt):
    """One slot carries a row, or few do: probabilities from 1 down to nothing."""
    st, n = store_with([300, 1000], 1, 1, 2, fmt, 230, gain=2.0)
    run(st, n, 1, 1, 2, 4, 9, mask=words(1, 9, 3), gain=6.0)
    run(st, n, 1, 1, 2, 4, 48, mask=words(1, 48, 3), gain=6.0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(3, 2), (40, 4), (64, 16)])
def test_rows_that_see_nothing(fmt, T, G):
    """An empty segment and a mask word of 0: the row gets 0, and gives nothing even where its
    query, output and gradient hold NaN."""
    st, n = store_with([0, 90], 1, 1, 2, fmt, 210)
    mask = words(1, T, 5)
    mask[0, 1] = 0
    if T < 64:
        mask |= -1 << T  # bits past the drafts
    x = step(st, 1, 1, 2, G, T, mask=mask)
    want = grads(st, x, 2)
    check(st, n, x, 2, want)
    assert not want["dq"][0, 0, 1, :G].float().any()
    for name in ("q", "dout", "out"):
        x[name][0, 0, 1, :G] = float("nan")
    got = grads(st, x, 2)
    for name in want:
        assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(4, 2), (32, 4), (64, 8)])
def test_unseen_drafts_do_not_touch_a_row(fmt, T, G):
    """Drafts that hold NaN and infinities: the rows that do not see them get bit for bit what
    they do without, and so do the drafts that those rows alone see."""
    st, n = store_with([200, 3], 1, 1, 2, fmt, 220)
    w = [(1 << t) | 1 if t % 2 else 1 for t in range(T)]
    mask = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in w]]).cuda()
    x = step(st, 1, 1, 2, G, T, mask=mask)
    want = grads(st, x, 2)
    check(st, n, x, 2, want)
    for i, value in enumerate((float("nan"), float("inf"))):
        x["k_new"][0, 0, 2, :, 3 + i] = value  # nobody sees draft 2
        x["v_new"][0, 0, 2, :, 9 + i] = value
    got = grads(st, x, 2)
    for name in want:
        a, b = (t[name][0, 0] if name in ("dk", "dv") else t[name] for t in (got, want))
        assert torch.equal(a, b), name
    assert not got["dk"][0, 0, 2].float().any() and not got["dv"][0, 0, 2].float().any()
    # draft 1 is seen by token 1 alone: only that token's gradient may change
    y = dict(x, v_new=x["v_new"].clone())
    y["v_new"][0, 0, 1, :, 5] = float("inf")
    got2 = grads(st, y, 2)
    rest = [t for t in range(T) if t != 1]
    assert torch.equal(got2["dq"][:, :, rest], got["dq"][:, :, rest])
    assert not torch.isfinite(got2["dq"][0, 0, 1].float()).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_nan_rows_stay_their_own(fmt):
    """A NaN in a query or an output's gradient reaches that row's gradient and what the row
    sees, not the other rows' gradients nor drafts it does not see."""
    T, G = 6, 2
    st, n = store_with([70], 1, 1, 1, fmt, 240)
    mask = torch.tensor([[1, 2, 4, 8, 16, 32]]).cuda()
    x = step(st, 1, 1, 1, G, T, mask=mask)
    want = grads(st, x, 1)
    for name in ("q", "dout"):
        y = dict(x, **{name: x[name].clone()})
        y[name][0, 0, 3, 1, 17] = float("nan")
        got = grads(st, y, 1)
        others = [t for t in range(T) if t != 3]
        assert torch.equal(got["dq"][:, :, others], want["dq"][:, :, others])
        assert torch.equal(got["dq"][0, 0, 3, 0], want["dq"][0, 0, 3, 0])
        assert torch.isnan(got["dq"][0, 0, 3, 1].float()).any()
        for d in ("dk", "dv"):
            assert torch.equal(got[d][:, :, others], want[d][:, :, others])
        assert torch.isnan(got["dk"][0, 0, 3].float()).any()
        assert torch.isnan(got["dk_store"].float()).any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_missing_pages(fmt):
    """Slots without a page are left out, as by the forward pass, and raise the status."""
    st, n = store_with([300, 200], 1, 1, 2, fmt, 250)
    st.table[0, 1], st.table[1, 0] = -1, st.k.shape[0]
    x, _ = run(st, n, 1, 1, 2, 4, 5)
    assert st.read_status() == ck.STATUS_STORE
    run(st, n, 1, 1, 2, 8, 40)


@pytest.mark.parametrize("fmt", FORMATS)
def test_odd_value_rows(fmt):
    """Rows of zeros and rows of very different sizes among the keys and values."""
    st, n = store_with([500], 1, 1, 1, fmt, 260)
    k, v = randn((1, 1, 64, 1, 128), 1), randn((1, 1, 64, 1, 128), 2)
    v[0, 0, ::3] = 0
    v[0, 0, 1::3] *= 2.0 ** 20
    k[0, 0, 5::7] = 0
    k[0, 0, 6::7] *= 2.0 ** -30
    ck.certkv_store_append(k, v, st, start=torch.tensor([100], dtype=torch.int32).cuda())
    st.counts.fill_(500)
    for T, G in ((1, 4), (33, 4), (64, 4)):
        run(st, n, 1, 1, 1, G, T)


@pytest.mark.parametrize("fmt", FORMATS)
def test_strides_of_every_argument(fmt):
    """Views of fused projections, layouts with heads before tokens, a broadcast gradient."""
    B, L, T, H, G = 2, 2, 9, 2, 3
    st, n = store_with([90, 200, 64, 5], B, L, H, fmt, 270)
    x = step(st, B, L, H, G, T)
    want = grads(st, x, H)

    def moved(t):  # [B][L][H][T][D] in memory
        return t.transpose(2, 3).contiguous().transpose(2, 3)

    y = {a: moved(b) if a in ("q", "k_new", "v_new", "out", "dout") else b for a, b in x.items()}
    fused = torch.full((B, L, T, H * G + 2 * H, 128), FILL, dtype=torch.bfloat16, device="cuda")
    outs = fused.split((H * G, H, H), dim=3)
    got = grads(st, y, H, dq=outs[0], dk_new=outs[1], dv_new=outs[2])
    for name in want:
        assert torch.equal(got[name], want[name]), name
    x["dout"] = x["dout"][:, :, :1].expand(B, L, T, H * G, 128)
    a = grads(st, x, H)
    x["dout"] = x["dout"].contiguous()
    b = grads(st, x, H)
    for name in want:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("fmt", FORMATS)
def test_parts_alone_and_repeats(fmt):
    """Each group of outputs alone is bit for bit what it is among the others; so is a repeat."""
    import ctypes
    B, L, H, G, T = 1, 1, 3, 4, 20
    st, n = store_with([700, 1, 130], B, L, H, fmt, 280)
    x = step(st, B, L, H, G, T)
    want = grads(st, x, H)
    again = grads(st, x, H)
    for name in want:
        assert torch.equal(again[name], want[name]), name
    alone = grads(st, x, H, pools=False)
    assert all(torch.equal(alone[a], want[a]) for a in alone)
    lib, s = ck.load_library(), st.struct()
    sh = ck.certkv_shape(B, L, H * G, H, 2, 128, 1)
    need = lib.certkv_tree_grad_workspace_bytes(ctypes.byref(sh), T)
    ws = ck.workspace(need, "cuda")
    r = {a: ctypes.byref(ck._rows(x[a], a)) for a in ("q", "k_new", "v_new", "out", "dout")}
    new = {a: torch.full_like(want[a], FILL) for a in want}
    d = {a: ctypes.byref(ck._rows(new[a], a)) for a in ("dq", "dk", "dv")}
    p = {a: new[a].data_ptr() for a in ("dk_store", "dv_store")}

    def call(dq=None, dk=None, dv=None, ks=None, vs=None):
        assert lib.certkv_tree_attn_grad(
            ctypes.byref(sh), T, r["q"], r["k_new"], r["v_new"], None, ctypes.byref(s), 0.0, r["out"],
            x["lse"].data_ptr(), r["dout"], None, dq, dk, dv, ks, vs, ws.data_ptr(), need, None) == ck.OK
        torch.cuda.synchronize()

    call(dq=d["dq"])
    call(dk=d["dk"], dv=d["dv"])
    call(ks=p["dk_store"], vs=p["dv_store"])
    for name in want:
        assert torch.equal(new[name], want[name]), name


def test_streams_graphs_and_a_shared_workspace():
    """Two captured calls that share a workspace, replayed on another stream with inputs that
    changed, equal direct calls."""
    B, L, H = 1, 2, 2
    cases = []
    side = torch.cuda.Stream()
    need = max(ck.certkv_tree_grad_workspace_bytes(B, L, H * G, H, T) for G, T in ((4, 3), (4, 40)))
    ws = ck.workspace(need, "cuda")
    for i, (fmt, G, T) in enumerate((("bf16", 4, 3), ("fp4", 4, 40))):
        st, n = store_with([400, 90], B, L, H, fmt, 300 + i)
        x = step(st, B, L, H, G, T, seed=i)
        outs = {a: torch.empty_like(x[b]) for a, b in (("dq", "q"), ("dk_new", "k_new"),
                                                       ("dv_new", "v_new"))}
        grads(st, x, H, ws=ws, **outs)
        cases.append((st, x, outs))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for st, x, outs in cases:
            grads(st, x, H, pools=False, ws=ws, **outs)
    for seed in (50, 60):
        for st, x, outs in cases:
            x["dout"].copy_(randn(tuple(x["dout"].shape), seed))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        for st, x, outs in cases:
            got = {a: b.clone() for a, b in outs.items()}
            want = grads(st, x, H, pools=False)
            assert torch.equal(got["dq"], want["dq"])
            assert torch.equal(got["dk_new"], want["dk"]) and torch.equal(got["dv_new"], want["dv"])


def test_two_calls_at_once():
    """Calls on two streams with a workspace each, over one store and over two, equal calls alone."""
    st, n = store_with([900, 90], 1, 2, 2, "fp8", 370)
    other, m = store_with([40, 700], 1, 2, 2, "bf16", 371)
    work = [(st, step(st, 1, 2, 2, 4, 40, seed=1)), (st, step(st, 1, 2, 2, 4, 7, seed=2)),
            (other, step(other, 1, 2, 2, 4, 40, seed=3)), (other, step(other, 1, 2, 2, 2, 20, seed=4))]
    want = [grads(s, x, 2) for s, x in work]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for a, b in ((0, 1), (0, 2), (1, 3), (2, 3)):
        got = {}
        for _ in range(4):
            for i, on in ((a, streams[0]), (b, streams[1])):
                with torch.cuda.stream(on):
                    got[i] = grads(work[i][0], work[i][1], 2)
        torch.cuda.synchronize()
        for i in (a, b):
            for name in want[i]:
                assert torch.equal(got[i][name], want[i][name]), (a, b, name)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("units,G,T", [(300, 4, 1), (300, 4, 5), (700, 2, 64), (40, 16, 64)])
def test_many_segments(fmt, units, G, T):
    counts = [0, 3, 64, 130, 1]
    st, n = store_with(counts, 1, 1, units, fmt, 310)
    run(st, n, 1, 1, units, G, T)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(64, 32), (63, 31), (64, 17), (17, 32)])
def test_most_rows(fmt, T, G):
    """As many query rows of a segment as there may be, and some fewer."""
    st, n = store_with([0, 129, 400], 1, 1, 3, fmt, 380)
    run(st, n, 1, 1, 3, G, T, mask=words(1, T, 8))
    run(st, n, 1, 1, 3, G, T, new=False, pools=False)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", [5, 40])
def test_broadcast_inputs(fmt, T):
    """Inputs that repeat along a dimension of stride 0: their gradients come whole, as those of
    copies."""
    st, n = store_with([200, 61], 2, 1, 2, fmt, 390)
    x = step(st, 2, 1, 2, 4, T, seed=5)
    x["dout"] = randn((2, 1, 1, 1, 128), 391).expand(2, 1, T, 8, 128)
    x["q"] = randn((1, 1, T, 8, 128), 392).expand(2, 1, T, 8, 128)
    x["k_new"] = randn((2, 1, 1, 2, 128), 393).expand(2, 1, T, 2, 128)
    x["out"] = ck.certkv_tree_attn(x["q"], st, hkv=2, k_new=x["k_new"], v_new=x["v_new"], lse=x["lse"])
    got = grads(st, x, 2)
    check(st, n, x, 2, got)
    y = dict(x, **{a: x[a].contiguous() for a in ("dout", "q", "k_new")})
    want = grads(st, y, 2)
    assert all(torch.equal(got[a], want[a]) for a in want)


def test_thousands_of_segments():
    """More than one pass of the scan over their tiles."""
    st, n = store_with([0, 3, 64, 130, 1, 200, 5], 1, 9, 1000, "bf16", 315)
    run(st, n, 1, 9, 1000, 1, 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 4), (32, 4), (64, 8)])
def test_long_segments_are_cut(fmt, T, G):
    """Segments that many blocks share."""
    st, n = store_with([20000, 37], 1, 1, 2, fmt, 320)
    run(st, n, 1, 1, 2, G, T)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(2, 4), (64, 8)])
def test_long_segments_without_drafts(fmt, T, G):
    st, n = store_with([20000, 37], 1, 1, 2, fmt, 325)
    run(st, n, 1, 1, 2, G, T, new=False, pools=False)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G,pools", [(4, 4, True), (40, 4, True), (4, 4, False)])
def test_nothing_live(fmt, T, G, pools):
    """Counts of nothing, below nothing and beyond the table; pages that are none."""
    st, n = store_with([0], 1, 1, 2, fmt, 340)
    run(st, n, 1, 1, 2, G, T, pools=pools)
    x, got = run(st, n, 1, 1, 2, G, T, new=False, pools=pools)
    assert not got["dq"].float().any()
    st, n = store_with([128, 64], 1, 1, 2, fmt, 341, room=0)
    want = run(st, n, 1, 1, 2, G, T, pools=pools)[1]
    st.counts[0] = 2 ** 31 - 1
    got = run(st, n, 1, 1, 2, G, T, pools=pools)[1]
    assert all(torch.equal(got[a], want[a]) for a in want)
    st.counts.fill_(-2 ** 31)
    run(st, [0, 0], 1, 1, 2, G, T, pools=pools)


@pytest.mark.parametrize("fmt", FORMATS)
def test_smallest_scale(fmt):
    """The least scale there is: logits are 0, and so are the gradients that it multiplies."""
    st, n = store_with([200, 70], 1, 1, 2, fmt, 350)
    for T in (6, 40):
        x, got = run(st, n, 1, 1, 2, 4, T, scale=2.0 ** -149)
        assert not got["dq"].float().any() and not got["dk"].float().any()
        x, got = run(st, n, 1, 1, 2, 4, T, scale=2.0 ** -149, pools=False)
        assert not got["dq"].float().any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(5, 4), (40, 4)])
def test_pools_beyond_32_bits(fmt, T, G):
    """Pages on both sides of offsets that 32 bits cannot hold: bit for bit what they give in a
    small pool."""
    st, n = store_with([300, 90], 1, 1, 2, fmt, 360)
    x = step(st, 1, 1, 2, G, T)
    want = grads(st, x, 2)
    old = st.k.shape[0]
    pages = 2 ** 32 // (st.k.element_size() * st.k[0].numel()) + 70
    far = [pages - 1 - 3 * i if i % 2 else pages - 60 - 5 * i for i in range(old)]
    assert len(set(far)) == old and min(far) < pages - 70 < max(far)
    at = torch.tensor(far, device="cuda")
    big = {}
    for name in ("k", "v", "k_scale", "v_scale", "k_group", "v_group"):
        t = getattr(st, name)
        if t is not None:
            big[name] = torch.empty((pages,) + t.shape[1:], dtype=t.dtype, device="cuda")
            big[name].view(torch.uint8)[at] = t.view(torch.uint8)
    table = at.int()[st.table.long()]
    large = ck.Store(table=table, counts=st.counts, format=fmt, status=st.status, **big)
    pools = [torch.empty((pages, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p in pools:
        p[at] = FILL
    got = dict(zip(("dq", "dk", "dv"), ck.certkv_tree_attn_grad(
        x["dout"], x["q"], large, x["out"], x["lse"], hkv=2, k_new=x["k_new"], v_new=x["v_new"],
        dk_store=pools[0], dv_store=pools[1])))
    got.update(dk_store=pools[0][at], dv_store=pools[1][at])
    for name in want:
        assert torch.equal(got[name], want[name]), name
    assert st.read_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_training_step_over_pages(fmt):
    """Pages reserved, slots mapped, rows appended, attended to and differentiated, captured
    together: the slots' gradients gathered by the map are those of the rows, step by step."""
    B, L, H, G, T = 2, 1, 2, 2, 30
    U = B * L * H
    st = ck.Store.empty(U, 4, fmt, pool_pages=16)
    pg = ck.certkv_pages_list(st)
    room = torch.full((B,), T, dtype=torch.int32, device="cuda")
    k, v = (randn((B, L, T, H, 128), 70 + i) for i in range(2))
    q, dout = (randn((B, L, T, H * G, 128), 72 + i) for i in range(2))
    lse, out, dq = torch.empty((B, L, T, H * G), device="cuda"), torch.empty_like(q), torch.empty_like(q)
    slots = torch.empty((U, T), dtype=torch.int32, device="cuda")
    pos = torch.empty((B, T), dtype=torch.int32, device="cuda")
    pools = [torch.full((16, 64, 128), FILL, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    wss = [ck.workspace(int(n), "cuda") for n in (
        ck.certkv_pages_workspace_bytes(st), ck.certkv_tree_workspace_bytes(B, L, H * G, H, T),
        ck.certkv_tree_grad_workspace_bytes(B, L, H * G, H, T))]

    def one():
        ck.certkv_pages_reserve(st, pg, room, ws=wss[0])
        ck.certkv_slot_map(st, T, batch=B, slots=slots, positions=pos)
        ck.certkv_store_append(k, v, st)
        ck.certkv_tree_attn(q, st, hkv=H, lse=lse, out=out, ws=wss[1])
        ck.certkv_tree_attn_grad(dout, q, st, out, lse, hkv=H, dq=dq, dk_store=pools[0],
                                 dv_store=pools[1], ws=wss[2])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one()
    for n in range(1, 5):  # 30, 60, 90 and 120 slots: pages end inside tiles
        for t, seed in ((k, 80), (v, 81), (q, 82), (dout, 83)):
            t.copy_(randn(tuple(t.shape), seed + 10 * n))
        graph.replay()
        torch.cuda.synchronize()
        assert st.counts.tolist() == [n * T] * U and st.read_status() == 0
        x = dict(q=q, dout=dout, out=out, lse=lse, k_new=None, v_new=None, mask=None, scale=0.0, dlse=None)
        check(st, [n * T] * U, x, H, dict(dq=dq, dk_store=pools[0], dv_store=pools[1]))
        new = slots.long()
        assert torch.equal(new.cpu(), torch.stack([st.table.cpu()[u].long()[torch.arange((n - 1) * T, n * T) // 64] * 64
                                                   + torch.arange((n - 1) * T, n * T) % 64 for u in range(U)]))
        rows = pools[0].view(-1, 128)[new]  # what a training step would hand on
        assert torch.isfinite(rows.float()).all() and not (rows == FILL).all(2).any()


def test_against_differences():
    """The change of a loss along random directions, from forward passes in 64 bits: the whole
    chain forward, then backward.  fp32 differences of bf16 passes would drown; the definition's
    forward pass in 64 bits is what is differentiated."""
    import drafts
    B, L, H, G, T = 1, 1, 1, 2, 4
    st, n = store_with([40], B, L, H, "bf16", 330)
    x = step(st, B, L, H, G, T)
    got = grads(st, x, H)
    f = {a: x[a].double().cpu().numpy() for a in ("q", "k_new", "v_new", "dout")}
    kv = [drafts.values(drafts.held(st, a)) for a in ("k", "v")]
    at = drafts.slots(st.table.cpu().numpy(), 0, 0, 40)

    def loss(q, k, v, ks, vs):
        total = 0.0
        for t in range(T):
            K, V = np.concatenate([ks[at], k[0, 0, :t + 1, 0]]), np.concatenate([vs[at], v[0, 0, :t + 1, 0]])
            z = q[0, 0, t] @ K.T / np.sqrt(128.0)
            p = np.exp(z - z.max(1, keepdims=True))
            total += (f["dout"][0, 0, t] * ((p / p.sum(1, keepdims=True)) @ V)).sum()
        return total

    args = [f["q"], f["k_new"], f["v_new"], kv[0], kv[1]]
    rng = np.random.default_rng(0)
    for i, name in enumerate(("dq", "dk", "dv", "dk_store", "dv_store")):
        g = got[name].double().cpu().numpy().reshape(args[i].shape)
        step_ = rng.standard_normal(args[i].shape)
        if name.endswith("_store"):
            live = np.zeros((len(args[i]), 1))
            live[at] = 1
            step_ *= live
            g = np.where(live > 0, g, 0.0)
        h = 1e-5
        up, down = ([a + s * h * step_ if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        # each element is off by 2^-8 of itself and as much of what is summed into it
        # (treegrad.py), `out` by 2^-8 in delta; the signs of a random direction are independent
        tol = 8 * 2.0 ** -8 * np.sqrt(((g * step_) ** 2).sum()) + 1e-3 * abs(slope)
        assert abs((g * step_).sum() - slope) <= tol, (name, (g * step_).sum(), slope, tol)
