"""Measured cases of the operators that verify drafted tokens over a paged, quantised store.

Three operators belong together here: rotary positions on the queries and keys of the drafted
tokens, the paged key/value store that the compressed cache and the accepted tokens are
quantised into and read back from, and attention of a tree of drafted tokens over that store.

`run` computes a case in one of two ways: with `own` false in elementary torch operations in
32 bits, with `own` true by the calls of this repository's package.  `exact` computes the same
outputs from the operators' definitions in 64 bits.
"""
import math

import torch

own = False

PAGE = 64     # slots of a page
D = 128       # head dimension
TINY = 2.0 ** -100  # rows whose largest element is below this are stored as zeros


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # q and k of eight sequences' drafted tokens, views of one fused projection
        dict(name="rope-step", op="rope", B=8, L=1, H=8, G=4, T=8, dim=128, layout="half",
             base=10000.0, factor=1.0, inverse=False, fused=True),
        # a whole prompt, half of each head rotated, long-context frequency ramp
        dict(name="rope-prompt", op="rope", B=1, L=1, H=8, G=4, T=32749, dim=64,
             layout="interleaved", base=500000.0, factor=4.0, inverse=False, fused=False),
        # a compressed 32-layer, 131072-token cache (budget 1/10) stored in 8 bits
        dict(name="load-fp8", op="load", B=1, L=32, H=8, slots=6553, reserve=64, format="fp8"),
        # the accepted drafts of eight sequences, all layers, after a verification step
        dict(name="append-step-fp8", op="append", B=8, L=32, H=8, T=8, format="fp8", tree=True),
        # an uncompressed 131071-token prompt of one layer written in 4 bits and read back
        dict(name="append-prompt-fp4", op="append", B=1, L=1, H=8, T=131071, format="fp4",
             tree=False),
        # a short window of every head read back for inspection
        dict(name="read-fp8", op="read", B=1, L=4, H=8, slots=4096, T=4091, format="fp8"),
        # one decode token over one layer's compressed 4096-token cache: latency counts
        dict(name="attn-step-bf16", op="attn", B=1, L=1, H=8, G=4, T=1, slots=409, format="bf16",
             tree=False, ragged=True, fused=False),
        # single tokens of eight sequences, four layers, 8 queries per key head
        dict(name="attn-decode-fp8", op="attn", B=8, L=4, H=8, G=8, T=1, slots=13107, format="fp8",
             tree=False, ragged=True, fused=False),
        # a 16-token draft tree over every layer of the compressed 131072-token cache
        dict(name="attn-tree-bf16", op="attn", B=1, L=32, H=8, G=4, T=16, slots=13107,
             format="bf16", tree=True, ragged=True, fused=False),
        # a 32-token tree for each of eight sequences, 64/8 heads, one layer
        dict(name="attn-tree-fp8", op="attn", B=8, L=1, H=8, G=8, T=32, slots=13107, format="fp8",
             tree=True, ragged=True, fused=True),
        # a 64-token tree over one layer's whole uncompressed cache in 4 bits
        dict(name="attn-tree-fp4-long", op="attn", B=1, L=1, H=8, G=4, T=64, slots=131072,
             format="fp4", tree=True, ragged=False, fused=False),
        # odd head counts and lengths, some heads with nothing stored
        dict(name="attn-odd-fp4", op="attn", B=3, L=2, H=5, G=3, T=7, slots=1001, format="fp4",
             tree=True, ragged=True, fused=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "load", "append", "read", "attn", "attn", "attn", "attn"])
    B, L, H = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 5, 32]), rng.choice([1, 2, 5, 8, 32])
    fmt = rng.choice(["bf16", "fp8", "fp4"])
    units = B * L * H
    if op == "rope":
        G = rng.choice([1, 3, 4, 8])
        T = _log(rng, 1, max(1, 32749 * 40 // (B * L * H * (G + 1))))
        return dict(op=op, B=B, L=L, H=H, G=G, T=T, dim=rng.choice([2, 32, 64, 96, 128]),
                    layout=rng.choice(["half", "interleaved"]),
                    base=rng.choice([10000.0, 500000.0]), factor=rng.choice([1.0, 2.0, 8.0]),
                    inverse=rng.random() < 0.3, fused=rng.random() < 0.5)
    most = 256 * 13107 // units
    if op == "load":
        return dict(op=op, B=B, L=L, H=H, slots=_log(rng, 2, min(131072, most // 2)),
                    reserve=rng.choice([0, 1, 64, 100]), format=fmt)
    if op == "append":
        tree = rng.random() < 0.5
        T = rng.randint(1, 64) if tree else _log(rng, 1, max(1, min(131071, most // 8)))
        return dict(op=op, B=B, L=L, H=H, T=T, format=fmt, tree=tree)
    if op == "read":
        slots = _log(rng, 1, min(65536, max(1, most // 4)))
        return dict(op=op, B=B, L=L, H=H, slots=slots, T=rng.randint(1, slots), format=fmt)
    G, T = rng.choice([1, 2, 3, 4, 8, 16]), _log(rng, 1, 64)
    # no more rows x slots, and no more slots, than the largest listed cases
    top = min(131072, most // 2, 8 * 131072 * 256 // (units * max(64, T * G)))
    return dict(op=op, B=B, L=L, H=H, G=G, T=T, slots=_log(rng, 1, max(1, top)), format=fmt,
                tree=T > 1 and rng.random() < 0.7, ragged=rng.random() < 0.6,
                fused=rng.random() < 0.5)


# ----------------------------------------------------------------- inputs --
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _counts(g, units, slots, ragged):
    """Slots of every head: the same for all, or spread as the budgets of a layer are
    (0.3 to 1.7 of the mean, and one head in sixteen with nothing)."""
    if not ragged:
        return torch.full((units,), slots, dtype=torch.int32, device="cuda")
    f = 0.3 + 1.4 * torch.rand(units, generator=g, device="cuda")
    c = torch.floor(f * slots).to(torch.int32)
    gone = torch.rand(units, generator=g, device="cuda") < 1.0 / 16
    return torch.where(gone, 0, c)


def _capacity(slots, ragged, more):
    """Pages of a head that hold its longest length and `more` further slots."""
    return -(-(int(1.7 * slots) + 1 + more if ragged else slots + more) // PAGE)


def _pool(fmt, pages):
    """An empty store of `pages` pages."""
    s = {"format": fmt, "pages": pages}
    for x in ("k", "v"):
        if fmt == "bf16":
            s[x] = torch.zeros((pages, PAGE, D), dtype=torch.bfloat16, device="cuda")
        elif fmt == "fp8":
            s[x] = torch.zeros((pages, PAGE, D), dtype=torch.float8_e4m3fn, device="cuda")
        else:
            s[x] = torch.zeros((pages, PAGE, D // 2), dtype=torch.uint8, device="cuda")
            s[x + "_group"] = torch.zeros((pages, PAGE, D // 16), dtype=torch.float8_e4m3fn,
                                          device="cuda")
        if fmt != "bf16":
            s[x + "_scale"] = torch.zeros((pages, PAGE), dtype=torch.float32, device="cuda")
    return s


def _shuffled_table(g, units, per_unit):
    """A page table whose pages lie in the pool in no order, as after many allocations."""
    return torch.randperm(units * per_unit, generator=g, device="cuda").to(torch.int32).view(
        units, per_unit)


def _filled(g, fmt, pages, heavy=None):
    """A store whose pages hold quantised rows; a few keys point along `heavy` [D]."""
    s = _pool(fmt, pages)
    for x in ("k", "v"):
        for p0 in range(0, pages, 16384):
            n = min(16384, pages - p0)
            rows = _randn(g, n, PAGE, D)
            if x == "k" and heavy is not None:
                rows[:, 7] = torch.where((torch.arange(n, device="cuda") % 8 == 0)[:, None],
                                         0.5 * heavy + rows[:, 7], rows[:, 7])
            for name, t in _encode(rows.to(torch.bfloat16), fmt).items():
                s[x + name].view(torch.uint8)[p0:p0 + n] = t.view(torch.uint8).view(
                    s[x + name].view(torch.uint8)[p0:p0 + n].shape)
    return s


def _parents(g, T):
    """A draft tree: every token's parent among the earlier ones (-1: the committed text)."""
    r = torch.rand(T, generator=g, device="cuda").cpu().tolist()
    return [min(i - 1, int(r[i] * (i + 1)) - 1) if i else -1 for i in range(T)]


def _tree(g, B, T):
    """Per sequence: 64-bit words, bit j of token i set where i sees j (its ancestors and itself)."""
    words = []
    for _ in range(B):
        seen = []
        for i, p in enumerate(_parents(g, T)):
            seen.append((seen[p] if p >= 0 else 0) | (1 << i))
        words.append([w - (1 << 64) if w >= 1 << 63 else w for w in seen])
    return torch.tensor(words, dtype=torch.int64, device="cuda")


def _projected(g, B, L, T, H, G, fused, gain=1.0):
    """q [B][L][T][H G][D], k, v [B][L][T][H][D]: views of one fused projection, or dense."""
    if fused:
        x = _randn(g, B, L, T, H * (G + 2), D).to(torch.bfloat16)
        q, k, v = x[..., :H * G, :], x[..., H * G:H * (G + 1), :], x[..., H * (G + 1):, :]
        q.mul_(gain)
        return q, k, v
    return ((gain * _randn(g, B, L, T, H * G, D)).to(torch.bfloat16),
            _randn(g, B, L, T, H, D).to(torch.bfloat16),
            _randn(g, B, L, T, H, D).to(torch.bfloat16))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, {"case": case}
    op, B, L, H = c["op"], c["B"], c["L"], c["H"]
    units = B * L * H
    if op == "rope":
        s["q"], s["k"], _ = _projected(g, B, L, c["T"], H, c["G"], c["fused"])
        first = torch.randint(0, 131072 - 32768, (B, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(c["T"], device="cuda")[None]).to(torch.int32)
    elif op == "load":
        mean = c["slots"]
        # `slots` a head, and as much again for the last head: the budgets of a layer differ
        n = torch.clamp(_counts(g, units, mean, True), min=1).view(B * L, H)
        n[:, -1] += H * (2 * mean) - n.sum(1, dtype=torch.int32)  # one budget for each layer
        n = n.view(units)
        total = B * L * H * 2 * mean
        s["total"] = total
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"),
                                  torch.cumsum(n, 0)])
        s["real"] = n - 1  # the last slot of a head is its tail slot
        s["pk"] = _randn(g, total, D).to(torch.bfloat16)
        s["pv"] = (_randn(g, total, D) * torch.exp(_randn(g, total, 1))).to(torch.bfloat16)
        s["max_pages"] = -(-(H * 2 * mean + c["reserve"]) // PAGE)
        s["store"] = _pool(c["format"], (total + units * c["reserve"]) // PAGE + 2 * units)
        s["store"]["table"] = torch.full((units, s["max_pages"]), -1, dtype=torch.int32,
                                         device="cuda")
        s["store"]["counts"] = torch.zeros(units, dtype=torch.int32, device="cuda")
    elif op == "append":
        T = c["T"]
        per = 4 + -(-T // PAGE)
        s["start"] = torch.randint(0, 4 * PAGE, (units,), generator=g, device="cuda").to(
            torch.int32)
        s["store"] = _pool(c["format"], units * per)
        s["store"]["table"] = _shuffled_table(g, units, per)
        s["store"]["counts"] = s["start"].clone()
        if c["tree"]:
            s["k"], s["v"] = (_randn(g, B, L, T, H, D).to(torch.bfloat16) for _ in range(2))
            s["accepted"] = torch.randint(1, T + 1, (B,), generator=g, device="cuda").to(
                torch.int32)
            order = torch.rand(B, T, generator=g, device="cuda").argsort(1)
            keep = torch.arange(T, device="cuda")[None] < s["accepted"][:, None]
            s["select"] = torch.where(keep, order, T).sort(1).values.clamp(max=T - 1).to(
                torch.int32)
        else:  # the layout of a prefilled cache: [B][L][H][T][D]
            s["k"], s["v"] = (_randn(g, B, L, H, T, D).to(torch.bfloat16).transpose(2, 3)
                              for _ in range(2))
            s["accepted"] = s["select"] = None
    elif op == "read":
        per = _capacity(c["slots"], False, 64)
        s["store"] = _filled(g, c["format"], units * per)
        s["store"]["table"] = _shuffled_table(g, units, per)
        s["store"]["counts"] = _counts(g, units, c["slots"], False)
        s["start"] = torch.randint(0, c["slots"] - c["T"] + 1, (units,), generator=g,
                                   device="cuda").to(torch.int32)
    else:
        T = c["T"]
        # logits that spread as trained heads' do: a few dozen slots carry most of a row
        s["q"], s["k"], s["v"] = _projected(g, B, L, T, H, c["G"], c["fused"], 2.5)
        per = _capacity(c["slots"], c["ragged"], T)
        heavy = s["q"].float().mean((0, 1, 2, 3))
        s["store"] = _filled(g, c["format"], units * per,
                             heavy * (math.sqrt(D) / heavy.norm().clamp_min(1e-6)))
        s["store"]["table"] = _shuffled_table(g, units, per)
        s["store"]["counts"] = _counts(g, units, c["slots"], c["ragged"])
        s["mask"] = _tree(g, B, T) if c["tree"] else None
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program keeps between calls of the package: plan, store, outputs and workspace."""
    from paper_2608_21541_gb300 import certkv as ck
    c = s["case"]
    if "store" in s:
        t = s["store"]
        s["handle"] = ck.Store(k=t["k"], v=t["v"], table=t["table"], counts=t["counts"],
                               format=c["format"], k_group=t.get("k_group"),
                               v_group=t.get("v_group"), k_scale=t.get("k_scale"),
                               v_scale=t.get("v_scale"))
    if c["op"] == "rope":
        s["plan"] = ck.certkv_rope_plan(c["dim"], layout=c["layout"], base=c["base"],
                                        scaling="ramp" if c["factor"] > 1 else "none",
                                        factor=c["factor"], original=8192, low=1.0, high=32.0,
                                        magnitude=_magnitude(c))
    elif c["op"] == "load":
        s["packed"] = ck.Packed(k=s["pk"], v=s["pv"], offsets=s["offsets"], real_counts=s["real"],
                                positions=torch.empty(s["total"], dtype=torch.int32,
                                                      device="cuda"))
        s["ws"] = ck.workspace(ck.certkv_store_workspace_bytes(len(s["real"])), "cuda")
    elif c["op"] == "attn":
        s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(s["q"].shape[:-1], dtype=torch.float32, device="cuda")
        s["ws"] = ck.workspace(ck.certkv_tree_workspace_bytes(c["B"], c["L"], c["H"] * c["G"],
                                                              c["H"], c["T"]), "cuda")


# -------------------------------------------------------------------- run --
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2608_21541_gb300 import certkv as ck
    c = s["case"]
    if c["op"] == "rope":
        return ck.certkv_rope(s["q"], s["positions"], s["plan"], s["k"], inverse=c["inverse"])
    st = s["handle"]
    if c["op"] == "load":
        ck.certkv_store_load(s["packed"], st, reserve=c["reserve"], ws=s["ws"])
        out = {"table": st.table, "counts": st.counts}
        if c["format"] != "fp4":
            return {**out, **_contents(s["store"])}
        most = min(s["max_pages"] * PAGE, 4 * c["slots"])
        return {**out, "rows": ck.certkv_store_read(st, most)}
    if c["op"] == "append":
        ck.certkv_store_append(s["k"], s["v"], st, select=s["select"], accepted=s["accepted"],
                               start=s["start"])
        if c["format"] != "fp4":
            return {"counts": st.counts, **_contents(s["store"])}
        return {"counts": st.counts, "rows": ck.certkv_store_read(st, c["T"], start=s["start"])}
    if c["op"] == "read":
        return ck.certkv_store_read(st, c["T"], start=s["start"])
    ck.certkv_tree_attn(s["q"], st, hkv=c["H"], k_new=s["k"], v_new=s["v"], mask=s["mask"],
                        out=s["out"], lse=s["lse"], ws=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _contents(t):
    return {n: t[n] for n in ("k", "v", "k_scale", "v_scale") if n in t}


# ------------------------------------------------------- the plain forms --
def _ramp(c):
    """theta_i in plain numbers: base^(-2i/dim), interpolated by `factor` where a frequency turns
    less than once over 8192 positions, kept above 32 turns, blended between."""
    th = [c["base"] ** (-2.0 * i / c["dim"]) for i in range(c["dim"] // 2)]
    if c["factor"] > 1:
        for i, t in enumerate(th):
            y = min(1.0, max(0.0, (8192 * t / (2 * math.pi) - 1.0) / (32.0 - 1.0)))
            th[i] = (1 - y) * t / c["factor"] + y * t
    return th


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0


def _rotate(x, cos, sin, c):
    half = c["layout"] == "half"
    r = x[..., :c["dim"]]
    r = r.unflatten(-1, (2, -1)) if half else r.unflatten(-1, (-1, 2)).transpose(-1, -2)
    a, b = r[..., 0, :], r[..., 1, :]
    y = torch.stack([a * cos - b * sin, a * sin + b * cos], -2)
    y = y.flatten(-2) if half else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., c["dim"]:]], -1)


def _encode(rows, fmt):
    """Quantised rows [..., D]: codes and scales by the store's definition, in 32 bits."""
    if fmt == "bf16":
        return {"": rows}
    x = rows.float()
    amax = x.abs().amax(-1, keepdim=True)
    top = 448.0 if fmt == "fp8" else 2688.0
    small = amax < TINY
    scale = torch.where(small, 1.0, amax / top)
    inv = torch.where(small, 0.0, top / amax)
    if fmt == "fp8":
        return {"": (x * inv).to(torch.float8_e4m3fn), "_scale": scale[..., 0]}
    xg = x.unflatten(-1, (D // 16, 16))
    gs = ((xg.abs().amax(-1) * inv) * (1.0 / 6.0)).to(torch.float8_e4m3fn)
    gf = gs.float()
    m = torch.where(gf > 0, inv * (1.0 / torch.where(gf > 0, gf, 1.0)), 0.0)
    y = xg * m[..., None]
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0))
    code = (code | ((y < 0).to(torch.uint8) << 3)).flatten(-2)
    return {"": code[..., 0::2] | (code[..., 1::2] << 4), "_group": gs, "_scale": scale[..., 0]}


def _decode(t, x, idx):
    """Rows of the pool at slots idx, in 32 bits."""
    rows = t[x].flatten(0, 1).view(torch.uint8)[idx]
    if t["format"] == "bf16":
        return rows.view(torch.bfloat16).float()
    scale = t[x + "_scale"].flatten()[idx][..., None]
    if t["format"] == "fp8":
        return rows.view(torch.float8_e4m3fn).float() * scale
    c = torch.stack([rows & 15, rows >> 4], -1).flatten(-2)
    mag = (c & 7).float()
    val = torch.where(mag < 2, mag * 0.5,
                      (2.0 + (c & 1)) * torch.exp2(torch.floor(mag * 0.5) - 2.0))
    val = torch.where(c >= 8, -val, val)
    gs = t[x + "_group"].flatten(0, 1).view(torch.uint8)[idx].view(torch.float8_e4m3fn).float()
    return (val.unflatten(-1, (-1, 16)) * gs[..., None]).flatten(-2) * scale


def _slot(table, s):
    """Pool slot of slot s [units][n] of every head."""
    page = torch.gather(table, 1, torch.clamp(s // PAGE, max=table.shape[1] - 1).long())
    return torch.clamp(page, min=0).long() * PAGE + (s % PAGE)


def _put(t, x, idx, rows):
    for name, val in _encode(rows, t["format"]).items():
        t[x + name].view(torch.uint8).view(t["pages"] * PAGE, -1)[idx] = val.contiguous().view(
            torch.uint8).view(*idx.shape, -1)


def _run_plain(s):
    c = s["case"]
    if c["op"] == "rope":
        return _plain_rope(s, c)
    return {"load": _plain_load, "append": _plain_append, "read": _plain_read,
            "attn": _plain_attn}[c["op"]](s, c, s["store"])


def _plain_rope(s, c):
    th = torch.tensor(_ramp(c), dtype=torch.float32, device="cuda")
    ang = s["positions"].float()[:, None, :, None, None] * th
    mag = _magnitude(c)
    cos, sin = torch.cos(ang) * mag, torch.sin(ang) * mag
    if c["inverse"]:
        cos, sin = cos / (mag * mag), -sin / (mag * mag)
    return (_rotate(s["q"].float(), cos, sin, c).to(torch.bfloat16),
            _rotate(s["k"].float(), cos, sin, c).to(torch.bfloat16))


def _plain_load(s, c, t):
    n = s["real"] + 1
    pages = (n + c["reserve"] + PAGE - 1) // PAGE
    first = torch.cumsum(pages, 0) - pages
    at = torch.arange(s["max_pages"], device="cuda")[None]
    t["table"].copy_(torch.where(at < pages[:, None], first[:, None] + at, -1))
    t["counts"].copy_(n)
    slot = torch.arange(s["total"], device="cuda")
    unit = torch.bucketize(slot, s["offsets"][1:], right=True)
    idx = first[unit].long() * PAGE + slot - s["offsets"][unit]
    _put(t, "k", idx, s["pk"])
    _put(t, "v", idx, s["pv"])
    out = {"table": t["table"], "counts": t["counts"]}
    if c["format"] != "fp4":
        return {**out, **_contents(t)}
    most = min(s["max_pages"] * PAGE, 4 * c["slots"])
    return {**out, "rows": _plain_rows(t, torch.zeros_like(t["counts"]), most)}


def _plain_rows(t, start, n):
    at = start[:, None] + torch.arange(n, device="cuda")[None]
    live = (at < t["counts"][:, None])[..., None]
    idx = _slot(t["table"], at)
    return tuple(torch.where(live, _decode(t, x, idx), 0.0).to(torch.bfloat16) for x in ("k", "v"))


def _plain_append(s, c, t):
    B, L, H, T = c["B"], c["L"], c["H"], c["T"]
    k, v = (s[x].transpose(2, 3).reshape(B, L * H, T, D) for x in ("k", "v"))
    at = s["start"][:, None] + torch.arange(T, device="cuda")[None]
    idx = _slot(t["table"], at)
    if s["select"] is None:
        t["counts"].copy_(s["start"] + T)
        _put(t, "k", idx, k.reshape(-1, T, D))
        _put(t, "v", idx, v.reshape(-1, T, D))
    else:
        t["counts"].copy_(s["start"] + s["accepted"].repeat_interleave(L * H, output_size=B * L * H))
        sel = s["select"].long()[:, None, :, None].expand(B, L * H, T, D)
        keep = (torch.arange(T, device="cuda")[None] < s["accepted"][:, None])
        keep = keep[:, None, :, None].expand(B, L * H, T, 1).reshape(-1, T, 1)
        for x, rows in (("k", k), ("v", v)):  # slots past the accepted ones keep what they hold
            new = _encode(torch.gather(rows, 2, sel).reshape(-1, T, D), t["format"])
            for name, val in new.items():
                pool = t[x + name].view(torch.uint8).view(t["pages"] * PAGE, -1)
                val = val.contiguous().view(torch.uint8).view(*idx.shape, -1)
                pool[idx] = torch.where(keep, val, pool[idx])
    if c["format"] != "fp4":
        return {"counts": t["counts"], **_contents(t)}
    return {"counts": t["counts"], "rows": _plain_rows(t, s["start"], T)}


def _plain_read(s, c, t):
    return _plain_rows(t, s["start"], c["T"])


def _plain_attn(s, c, t):
    B, L, H, G, T = c["B"], c["L"], c["H"], c["G"], c["T"]
    U, S = B * L * H, t["table"].shape[1] * PAGE
    q = s["q"].unflatten(3, (H, G)).permute(0, 1, 3, 2, 4, 5).reshape(U, T * G, D).float()
    kn, vn = (s[x].transpose(2, 3).reshape(U, T, D).float() for x in ("k", "v"))
    at = torch.arange(S, device="cuda")[None].expand(U, S)
    idx = _slot(t["table"], at)
    x = torch.cat([q @ _decode(t, "k", idx).transpose(1, 2), q @ kn.transpose(1, 2)], -1)
    x = x * (1.0 / math.sqrt(D))
    j = torch.arange(T, device="cuda")
    if s["mask"] is None:
        sees = (j[None, :] <= j[:, None])[None].expand(B, T, T)
    else:
        sees = (s["mask"][..., None] >> j) & 1 > 0
    sees = sees[:, None, :, None].expand(B, L * H, T, G, T).reshape(U, T * G, T)
    live = (at < t["counts"][:, None])[:, None].expand(U, T * G, S)
    x = torch.where(torch.cat([live, sees], -1), x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    l = p.sum(-1, keepdim=True)
    o = p[..., :S] @ _decode(t, "v", idx) + p[..., S:] @ vn
    o = torch.where(l > 0, o / l, 0.0)
    o = o.view(B, L, H, T, G, D).permute(0, 1, 3, 2, 4, 5).reshape(B, L, T, H * G, D)
    lse = (m + torch.log(l)).view(B, L, H, T, G).permute(0, 1, 3, 2, 4).reshape(B, L, T, H * G)
    return {"out": o.to(torch.bfloat16), "lse": lse}


# ------------------------------------------------------------------- work --
ROW_BYTES = {"bf16": 2 * D, "fp8": D + 4, "fp4": D // 2 + D // 16 + 4}


def work(case):
    c = case
    units = c["B"] * c["L"] * c["H"]
    if c["op"] == "rope":
        rows = units * (c["G"] + 1) * c["T"]
        return {"bytes": rows * 4 * D + 4 * c["B"] * c["T"], "flops": 3 * c["dim"] * rows}
    row = 2 * ROW_BYTES[c["format"]]
    if c["op"] == "load":
        n = units * 2 * c["slots"]
        back = min(2 * units * c["slots"], n) * 4 * D if c["format"] == "fp4" else 0
        return {"bytes": n * (4 * D + row) + back, "flops": 0}
    if c["op"] == "append":
        n = units * (c["T"] / 2 if c["tree"] else c["T"])
        back = n * (row + 4 * D) if c["format"] == "fp4" else 0
        return {"bytes": n * (4 * D + row) + back, "flops": 0}
    if c["op"] == "read":
        return {"bytes": units * c["T"] * (4 * D + row), "flops": 0}
    rows = units * c["G"] * c["T"]
    slots = units * c["slots"] * (15.0 / 16 if c["ragged"] else 1.0)
    return {"bytes": slots * row + rows * 4 * D + units * c["T"] * 4 * D,
            "flops": 4.0 * D * c["T"] * c["G"] * (slots + units * c["T"])}


# ----------------------------------------------------------------- 64 bits --
def _grid(fmt):
    """The values of the 8-bit (4 exponent, 3 mantissa bits) or 4-bit (2, 1) code, from their bits."""
    if fmt == "fp4":
        return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6],
                            dtype=torch.float64, device="cuda")
    vals = []
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        v = math.ldexp(8 + f, e - 10) if e else math.ldexp(f, -9)
        vals.append((-v if b & 128 else v) if (b & 127) != 127 else math.nan)
    return torch.tensor(vals, dtype=torch.float64, device="cuda")


def _nearest(y, fmt):
    """y rounded to the values of a code, ties to the even mantissa, beyond the largest to it."""
    man, low, top = (3, -6, 448.0) if fmt == "fp8" else (1, 0, 6.0)
    _, e = torch.frexp(y)
    step = torch.exp2((torch.clamp(e - 1, min=low) - man).double())
    return torch.clamp(torch.round(y / step) * step, -top, top)


def _stored64(rows, fmt):
    """The values rows [n][D] stand for once stored, in 64 bits, and (codes' values, scales)."""
    x = rows.double()
    if fmt == "bf16":
        return x, x, None
    top = 448.0 if fmt == "fp8" else 2688.0
    amax = x.abs().amax(-1, keepdim=True)
    r = torch.where(amax < TINY, 0.0, top / amax)
    scale = torch.where(amax < TINY, 1.0, amax / top)
    if fmt == "fp8":
        codes = _nearest(x * r, "fp8")
    else:
        xg = x.unflatten(-1, (-1, 16))
        gs = _nearest(xg.abs().amax(-1, keepdim=True) * r[..., None] / 6.0, "fp8")
        m = torch.where(gs > 0, r[..., None] / torch.where(gs > 0, gs, 1.0), 0.0)
        codes = (_nearest(xg * m, "fp4") * gs).flatten(-2)
    return codes * scale, codes, scale[..., 0]


def _held64(t, x, slots):
    """Rows of the pool at `slots` [n], in 64 bits."""
    pages, at = slots // PAGE, slots % PAGE
    if t["format"] == "bf16":
        return t[x][pages, at].double()
    raw = t[x].view(torch.uint8)[pages, at].long()
    scale = t[x + "_scale"][pages, at].double()[:, None]
    if t["format"] == "fp8":
        return _grid("fp8")[raw] * scale
    val = _grid("fp4")[torch.stack([raw & 15, raw >> 4], -1).reshape(len(slots), D)]
    gs = _grid("fp8")[t[x + "_group"].view(torch.uint8)[pages, at].long()]
    return val * gs.repeat_interleave(16, dim=1) * scale


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return _exact_rope(s, c)
    if c["op"] == "attn":
        return _exact_attn(s, c, s["store"])
    return _exact_store(s, c, s["store"])


def _exact_rope(s, c):
    n = c["dim"] // 2
    th = torch.tensor(_ramp(c), dtype=torch.float64, device="cuda")
    ang = s["positions"].double()[:, None, :, None, None] * th * (-1 if c["inverse"] else 1)
    mag = 1.0 / _magnitude(c) if c["inverse"] else _magnitude(c)
    got = []
    for x in (s["q"], s["k"]):
        y = x.double()
        i = torch.arange(n, device="cuda")
        ia, ib = (i, i + n) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.polar(torch.full_like(ang, mag), ang) * torch.complex(y[..., ia], y[..., ib])
        y[..., ia], y[..., ib] = z.real, z.imag
        got.append(y)
    return tuple(got)


def _exact_store(s, c, t):
    B, L, H = c["B"], c["L"], c["H"]
    U, fmt = B * L * H, c["format"]
    if c["op"] == "read":
        got = []
        for x in ("k", "v"):
            rows = torch.zeros((U, c["T"], D), dtype=torch.float64, device="cuda")
            for u in range(U):
                at = int(s["start"][u]) + torch.arange(c["T"], device="cuda")
                at = at[at < int(t["counts"][u])]
                rows[u, :len(at)] = _held64(t, x, t["table"][u, at // PAGE].long() * PAGE
                                            + at % PAGE)
            got.append(rows)
        return tuple(got)
    if U * c.get("T", 0) * D > 1 << 30 or c["op"] == "load" and s["total"] * D > 1 << 30:
        return None
    # the written rows of every head, in order, and the pool slots they go to
    first, moved, src = 0, [], {"k": [], "v": []}
    for u in range(U):
        b, l, h = u // (L * H), u // H % L, u % H
        if c["op"] == "load":
            lo, hi = int(s["offsets"][u]), int(s["offsets"][u + 1])
            src["k"].append(s["pk"][lo:hi])
            src["v"].append(s["pv"][lo:hi])
            moved.append(first * PAGE + torch.arange(hi - lo, device="cuda"))
            first += -(-(hi - lo + c["reserve"]) // PAGE)
            continue
        n = c["T"] if s["accepted"] is None else int(s["accepted"][b])
        pick = slice(0, n) if s["select"] is None else s["select"][b, :n].long()
        at = int(s["start"][u]) + torch.arange(n, device="cuda")
        for x in ("k", "v"):
            src[x].append(s[x][b, l, :, h][pick])
        moved.append(t["table"][u, at // PAGE].long() * PAGE + at % PAGE)
    to = torch.cat(moved)
    got = {"table": None, "counts": None} if c["op"] == "load" else {"counts": None}
    if fmt == "fp4":
        if c["op"] == "load":
            most = min(s["max_pages"] * PAGE, 4 * c["slots"])
            live = [min(len(m), most) for m in moved]
        else:
            most, live = c["T"], [len(m) for m in moved]
        rows = []
        for x in ("k", "v"):
            y = torch.zeros((U, most, D), dtype=torch.float64, device="cuda")
            for u in range(U):
                y[u, :live[u]] = _stored64(src[x][u][:live[u]], fmt)[0]
            rows.append(y)
        return {**got, "rows": tuple(rows)}
    for x in ("k", "v"):
        _, codes, scale = _stored64(torch.cat(src[x]), fmt)
        pool = torch.zeros((t["pages"] * PAGE, D), dtype=torch.float64, device="cuda")
        pool[to] = codes
        got[x] = pool.view(t["pages"], PAGE, D)
        if scale is not None:
            pool = torch.zeros(t["pages"] * PAGE, dtype=torch.float64, device="cuda")
            pool[to] = scale
            got[x + "_scale"] = pool.view(t["pages"], PAGE)
    return got


def _exact_attn(s, c, t):
    B, L, H, G, T = c["B"], c["L"], c["H"], c["G"], c["T"]
    out = torch.zeros((B, L, T, H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, L, T, H * G), -math.inf, dtype=torch.float64, device="cuda")
    counts = t["counts"].cpu().tolist()
    words = None if s["mask"] is None else s["mask"].cpu().tolist()
    unseen = [torch.tensor([[j > i if words is None else not words[b][i] >> j & 1
                             for j in range(T)] for i in range(T)], device="cuda")
              for b in range(B)]
    for u in range(B * L * H):
        b, l, h = u // (L * H), u // H % L, u % H
        at = torch.arange(counts[u], device="cuda")
        slots = t["table"][u, at // PAGE].long() * PAGE + at % PAGE
        k = torch.cat([_held64(t, "k", slots), s["k"][b, l, :, h].double()])
        v = torch.cat([_held64(t, "v", slots), s["v"][b, l, :, h].double()])
        q = s["q"][b, l, :, h * G:(h + 1) * G].double()  # [T][G][D]
        hide = torch.zeros((T, 1, counts[u] + T), dtype=torch.bool, device="cuda")
        hide[:, 0, counts[u]:] = unseen[b]
        x = ((q.reshape(T * G, D) @ k.T) / math.sqrt(D)).view(T, G, -1)
        x = x.masked_fill(hide, -math.inf)
        lse[b, l, :, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
        out[b, l, :, h * G:(h + 1) * G] = (torch.softmax(x, -1).view(T * G, -1) @ v).view(T, G, D)
    return {"out": out, "lse": lse}
