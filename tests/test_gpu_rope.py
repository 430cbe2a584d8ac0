"""Rotary positions against the rotation in 64 bits.  Bound: bf16 rounding of the
result (half an ulp, 2^-8 of it) and fp32 angles (2^-20 of the pair's magnitude)."""
import math

import numpy as np
import pytest
import torch

import drafts
from paper_2608_21541_gb300 import certkv as ck

pytestmark = pytest.mark.gpu


def reference(x, pos, dim, layout, base, mag=1.0, inverse=False, theta=None):
    y = x.double().cpu().numpy().copy()
    n = dim // 2
    i = np.arange(n)
    th = base ** (-2.0 * i / dim) if theta is None else theta
    ang = pos.cpu().numpy().astype(np.float64)[:, None, :, None, None] * th
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    c, s, m = np.cos(ang), np.sin(ang) * (-1 if inverse else 1), 1 / mag if inverse else mag
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = m * (xa * c - xb * s), m * (xa * s + xb * c)
    pair = m * np.sqrt(xa ** 2 + xb ** 2)
    tol = np.zeros(y.shape)
    tol[..., a], tol[..., b] = pair, pair
    return y, 2.0 ** -8 * np.abs(y) * (np.arange(128) < dim) + 2.0 ** -20 * tol


def check(got, ref):
    d = np.abs(got.double().cpu().numpy() - ref[0])
    assert (d <= ref[1] * 1.001).all(), np.max(d / np.maximum(ref[1], 1e-30))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim", [2, 6, 8, 64, 96, 126, 128])
@pytest.mark.parametrize("B,L,T,Hq,H", [(1, 1, 1, 1, 1), (2, 3, 5, 12, 4), (1, 2, 67, 5, 5)])
def test_matches_the_rotation(layout, dim, B, L, T, Hq, H):
    q, k = drafts.randn((B, L, T, Hq, 128), 1), drafts.randn((B, L, T, H, 128), 2)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-5, 1 << 20, (B, T), generator=g, dtype=torch.int32).cuda()
    plan = ck.certkv_rope_plan(dim, layout=layout, base=10000.0)
    qo, ko = ck.certkv_rope(q, pos, plan, k)
    check(qo, reference(q, pos, dim, layout, 10000.0))
    check(ko, reference(k, pos, dim, layout, 10000.0))
    # queries alone, in place: the same bits
    q2 = q.clone()
    assert ck.certkv_rope(q2, pos, plan, out=q2) is q2
    assert torch.equal(q2, qo)


@pytest.mark.parametrize("kind,factor", [("linear", 4.0), ("ntk", 8.0), ("ramp", 8.0)])
def test_scaled_frequencies_and_magnitude(kind, factor):
    dim, base, n = 128, 500000.0, 64
    i = np.arange(n)
    th = base ** (-2.0 * i / dim)
    if kind == "linear":
        th = th / factor
    elif kind == "ntk":
        th = (base * factor ** (dim / (dim - 2))) ** (-2.0 * i / dim)
    else:
        gam = np.clip((8192 * th / (2 * math.pi) - 1.0) / 31.0, 0, 1)
        th = (1 - gam) * th / factor + gam * th
    mag = 0.1 * math.log(factor) + 1.0
    plan = ck.certkv_rope_plan(dim, base=base, scaling=kind, factor=factor, magnitude=mag)
    q = drafts.randn((1, 1, 9, 3, 128), 4)
    pos = torch.arange(9, dtype=torch.int32).view(1, 9).cuda() * 14563
    ref = reference(q, pos, dim, "half", base, mag, theta=th)
    check(ck.certkv_rope(q, pos, plan), (ref[0], ref[1] * 1.01))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_positions_of_any_size_keep_their_angle(layout):
    """Position 2^31 - 1: a float product of position and frequency would be off by
    whole turns."""
    q = drafts.randn((1, 1, 4, 2, 128), 5)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 16777217 * 3]], dtype=torch.int32,
                       device="cuda")
    plan = ck.certkv_rope_plan(128, layout=layout)
    ref, tol = reference(q, pos, 128, layout, 10000.0)
    # the frequency itself is held to 2^-48, which 2^31 turns carry to 2^-17
    pair = np.abs(q.double().cpu().numpy()).max() * 2
    check(ck.certkv_rope(q, pos, plan), (ref, tol + 2.0 ** -14 * pair))


def test_inverse_undoes_and_is_the_gradient():
    """inverse = the transpose for magnitude 1: <R x, y> = <x, R' y>, checked against
    finite differences of the 64-bit rotation and by a round trip."""
    plan = ck.certkv_rope_plan(64, layout="interleaved")
    x, y = drafts.randn((1, 1, 6, 2, 128), 6), drafts.randn((1, 1, 6, 2, 128), 7)
    pos = (torch.arange(6, dtype=torch.int32) * 1001).view(1, 6).cuda()
    back = ck.certkv_rope(y, pos, plan, inverse=True)
    check(back, reference(y, pos, 64, "interleaved", 10000.0, inverse=True))
    # d/dx_j <R x, y> by central differences of the definition (linear: exact)
    yd = y.double().cpu().numpy()
    for j in (0, 1, 62, 63, 64, 127):
        e = torch.zeros_like(x)
        e[..., j] = 0.5
        up, dn = (reference(x.double() + s * e.double(), pos, 64, "interleaved", 10000.0)[0]
                  for s in (1, -1))
        diff = ((up - dn) * yd).sum(-1)
        got = back.double().cpu().numpy()[..., j]
        assert np.abs(diff - got).max() <= 2.0 ** -8 * np.abs(diff).max() + 1e-5
    there = ck.certkv_rope(x, pos, ck.certkv_rope_plan(128, magnitude=1.5))
    again = ck.certkv_rope(there, pos, ck.certkv_rope_plan(128, magnitude=1.5), inverse=True)
    d = (again.double() - x.double()).abs().max()
    assert d <= 2.0 ** -7 * x.double().abs().max() * 2  # two roundings of a turned pair


def test_views_and_untouched_elements():
    """Views of a fused projection, a head-major output, and elements past dim bit for
    bit, NaN and infinities among them."""
    B, L, T, Hq, H = 2, 2, 7, 8, 2
    x = drafts.randn((B, L, T, Hq + 2 * H, 128), 8)
    x[..., 40] = float("nan")
    x[..., 41] = float("inf")
    q, k = x[..., :Hq, :], x[..., Hq:Hq + H, :]
    pos = torch.arange(B * T, dtype=torch.int32).view(B, T).cuda() * 313
    for layout in ("half", "interleaved"):
        for dim in (32, 38):
            plan = ck.certkv_rope_plan(dim, layout=layout)
            ko = torch.empty((B, L, H, T, 128), dtype=torch.bfloat16, device="cuda").transpose(2, 3)
            qo, _ = ck.certkv_rope(q, pos, plan, k, k_out=ko)
            for got, src in ((qo, q), (ko, k)):
                bits = got.contiguous().view(torch.int16)
                assert torch.equal(bits[..., dim:], src.contiguous().view(torch.int16)[..., dim:])
                clean = src.clone()
                clean[..., 40:42] = 0
                ref, tol = reference(clean, pos, dim, layout, 10000.0)
                d = np.abs(got[..., :dim].double().cpu().numpy() - ref[..., :dim])
                assert (d <= tol[..., :dim] * 1.001).all()


def test_other_stream_and_graph():
    q = drafts.randn((1, 1, 8, 4, 128), 9)
    pos = torch.arange(8, dtype=torch.int32).view(1, 8).cuda()
    plan = ck.certkv_rope_plan()
    want = ck.certkv_rope(q, pos, plan)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = ck.certkv_rope(q, pos, plan, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.certkv_rope(q, pos, plan, out=out)
    pos += 5
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ck.certkv_rope(q, pos, plan))
