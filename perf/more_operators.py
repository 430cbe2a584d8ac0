"""Measured cases of the operators that keep a paged store's pages on the GPU and that train over it.

Two sets belong together here around the store that certkv_tree_attn reads: its pages (the free
list, pages handed out and taken back from request lengths, the slot map and positions of a
step), and the gradients of attention over it, which recompute the probabilities from the
log-sum-exp of the forward pass.

`run` computes a case in one of two ways: with `own` false in elementary torch operations in
32 bits, with `own` true by the calls of this repository's package.  `exact` computes the
gradients from their definition in 64 bits; everything else is whole numbers.
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
        # the free pages of a serving process, found again from its page table
        dict(name="list-serve", op="list", B=64, L=32, H=8, slots=1000, room=64),
        # room for eight sequences' drafts in one layer's store: latency counts
        dict(name="reserve-step", op="reserve", B=8, L=1, H=8, slots=409, room=16),
        # the same before every step of 64 sequences, all layers: what was not accepted goes back,
        # room for the next 64 drafts is taken
        dict(name="reserve-serve", op="reserve", B=64, L=32, H=8, slots=1000, room=64),
        # a finished 131072-token sequence's pages taken back and given to the next, all layers
        dict(name="reserve-prompt", op="reserve", B=1, L=32, H=8, slots=0, room=131072),
        # where 64 drafts of eight sequences go in every layer, and their depths in the draft trees
        dict(name="map-step", op="map", B=8, L=32, H=8, slots=1000, T=64, tree=True, ragged=True),
        # where a 131071-token prompt goes
        dict(name="map-prompt", op="map", B=1, L=32, H=8, slots=0, T=131071, tree=False,
             ragged=False),
        # one token over one layer's compressed 4096-token cache: latency counts
        dict(name="grad-step-bf16", op="grad", B=1, L=1, H=8, G=4, T=1, slots=409, format="bf16",
             tree=False, ragged=True, fused=False, pools=False),
        # every layer of a compressed 131072-token cache refined by 16 tokens' gradients
        dict(name="grad-refine-bf16", op="grad", B=1, L=32, H=8, G=4, T=16, slots=13107,
             format="bf16", tree=False, ragged=True, fused=False, pools=True),
        # a drafter trained on 32-token trees of eight sequences, 64/8 heads, one layer
        dict(name="grad-tree-fp8", op="grad", B=8, L=1, H=8, G=8, T=32, slots=13107, format="fp8",
             tree=True, ragged=True, fused=True, pools=False),
        # 64-token trees over one layer's whole uncompressed cache in 4 bits
        dict(name="grad-tree-fp4-long", op="grad", B=1, L=1, H=8, G=4, T=64, slots=131072,
             format="fp4", tree=True, ragged=False, fused=False, pools=False),
        # one layer's cache refined by 64 tokens of 128 query heads
        dict(name="grad-rows-bf16", op="grad", B=1, L=1, H=8, G=16, T=64, slots=32768,
             format="bf16", tree=False, ragged=False, fused=False, pools=True),
        # odd head counts and lengths, heads with nothing stored, a padding token that sees nothing
        dict(name="grad-odd-fp4", op="grad", B=3, L=2, H=5, G=3, T=7, slots=1001, format="fp4",
             tree=True, ragged=True, fused=True, pools=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["list", "reserve", "map", "grad", "grad", "grad", "grad", "grad"])
    B, L, H = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 5, 32]), rng.choice([1, 2, 5, 8, 32])
    units = B * L * H
    if op in ("list", "reserve"):
        B = rng.choice([1, 3, 8, 64]) if L * H <= 256 else 1
        most = 16384 * 2048 // (B * L * H)
        return dict(op=op, B=B, L=L, H=H, slots=_log(rng, 1, min(65536, most)),
                    room=_log(rng, 1, min(65536, most)))
    if op == "map":
        tree = rng.random() < 0.5
        T = rng.randint(1, 64) if tree else _log(rng, 1, min(131071, 33554176 // units))
        return dict(op=op, B=B, L=L, H=H, slots=_log(rng, 1, 8192), T=T, tree=tree,
                    ragged=rng.random() < 0.5)
    fmt, pools = rng.choice(["bf16", "fp8", "fp4"]), rng.random() < 0.4
    G, T = rng.choice([1, 2, 3, 4, 8, 16]), _log(rng, 1, 64)
    # no more rows x slots, and no more slots, than the largest listed cases
    top = min(131072, 256 * 13107 // units // 2, 8 * 131072 * 256 // (units * max(64, T * G)))
    return dict(op=op, B=B, L=L, H=H, G=G, T=T, slots=_log(rng, 1, max(1, top)), format=fmt,
                tree=T > 1 and rng.random() < 0.6, ragged=rng.random() < 0.6,
                fused=rng.random() < 0.5, pools=pools)


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


def _filled(g, fmt, pages, heavy):
    """A store whose pages hold quantised rows; a few keys point along `heavy` [D]."""
    s = _pool(fmt, pages)
    for x in ("k", "v"):
        for p0 in range(0, pages, 16384):
            n = min(16384, pages - p0)
            rows = _randn(g, n, PAGE, D)
            if x == "k":
                rows[:, 7] = torch.where((torch.arange(n, device="cuda") % 8 == 0)[:, None],
                                         0.5 * heavy + rows[:, 7], rows[:, 7])
            for name, t in _encode(rows.to(torch.bfloat16), fmt).items():
                s[x + name].view(torch.uint8)[p0:p0 + n] = t.view(torch.uint8).view(
                    s[x + name].view(torch.uint8)[p0:p0 + n].shape)
    return s


def _tree(g, B, T, padding=False):
    """Per sequence: 64-bit words, bit j of token i set where i sees j (its ancestors and
    itself); with `padding` the last token of every sequence sees nothing."""
    words = []
    for _ in range(B):
        r = torch.rand(T, generator=g, device="cuda").cpu().tolist()
        seen = []
        for i in range(T):
            p = min(i - 1, int(r[i] * (i + 1)) - 1) if i else -1
            seen.append((seen[p] if p >= 0 else 0) | (1 << i))
        if padding:
            seen[-1] = 0
        words.append([w - (1 << 64) if w >= 1 << 63 else w for w in seen])
    return torch.tensor(words, dtype=torch.int64, device="cuda")


def _projected(g, B, L, T, H, G, fused):
    """q [B][L][T][H G][D], k, v [B][L][T][H][D]: views of one fused projection, or dense."""
    if fused:
        x = _randn(g, B, L, T, H * (G + 2), D).to(torch.bfloat16)
        q, k, v = x[..., :H * G, :], x[..., H * G:H * (G + 1), :], x[..., H * (G + 1):, :]
        q.mul_(2.5)
        return q, k, v
    return ((2.5 * _randn(g, B, L, T, H * G, D)).to(torch.bfloat16),
            _randn(g, B, L, T, H, D).to(torch.bfloat16),
            _randn(g, B, L, T, H, D).to(torch.bfloat16))


def _table(g, units, per_unit, pool, held):
    """A page table whose pages lie in the pool in no order, as after many allocations: held[u]
    pages a row, -1 behind them; and the pages left over, in no order either."""
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    first = torch.cumsum(held, 0) - held
    at = torch.arange(per_unit, device="cuda")[None]
    mine = at < held[:, None]
    table = torch.where(mine, order[torch.clamp(first[:, None] + at, max=pool - 1)], -1)
    return table.to(torch.int32).contiguous(), order[int(held.sum()):]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, {"case": case}
    op, B, L, H = c["op"], c["B"], c["L"], c["H"]
    units = B * L * H
    if op in ("list", "reserve"):
        n = _counts(g, units, c["slots"], True)
        rooms = torch.full((B,), c["room"], dtype=torch.int32, device="cuda")
        if B > 1:  # sequences draft differently many tokens
            rooms = torch.randint(1, c["room"] + 1, (B,), generator=g, device="cuda").to(torch.int32)
        most = _capacity(c["slots"], True, c["room"])
        held = (n + PAGE - 1) // PAGE
        need = (n + rooms.repeat_interleave(L * H, output_size=units) + PAGE - 1) // PAGE
        pool = units * most
        if op == "list":
            held = need
        table, left = _table(g, units, most, pool, held)
        s["store"] = {"format": "bf16", "pages": pool, "table": table, "counts": n}
        s["free"] = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
        s["free"][:len(left)] = left
        s["n_free"] = torch.tensor([len(left)], dtype=torch.int32, device="cuda")
        s["held"] = held.to(torch.int32)
        s["rooms"], s["no_room"] = rooms, torch.zeros_like(rooms)
    elif op == "map":
        n = _counts(g, units, c["slots"], c["ragged"])
        per = _capacity(c["slots"], c["ragged"], c["T"])
        table, _ = _table(g, units, per, units * per,
                          torch.full((units,), per, device="cuda"))
        s["store"] = {"format": "bf16", "pages": units * per, "table": table, "counts": n}
        # sequences bring differently many rows
        s["rows"] = torch.full((B,), c["T"], dtype=torch.int32, device="cuda")
        if c["ragged"]:
            s["rows"] = torch.randint(0, c["T"] + 1, (B,), generator=g, device="cuda").to(
                torch.int32)
        s["base"] = torch.randint(0, 131072, (B,), generator=g, device="cuda").to(torch.int32)
        s["mask"] = _tree(g, B, c["T"]) if c["tree"] else None
    else:
        T = c["T"]
        # logits that spread as trained heads' do: a few dozen slots carry most of a row
        s["q"], s["k"], s["v"] = _projected(g, B, L, T, H, c["G"], c["fused"])
        per = _capacity(c["slots"], c["ragged"], T)
        heavy = s["q"].float().mean((0, 1, 2, 3))
        s["store"] = _filled(g, c["format"], units * per,
                             heavy * (math.sqrt(D) / heavy.norm().clamp_min(1e-6)))
        s["store"]["table"], _ = _table(g, units, per, units * per,
                                        torch.full((units,), per, device="cuda"))
        s["store"]["counts"] = _counts(g, units, c["slots"], c["ragged"])
        s["mask"] = _tree(g, B, T, c["ragged"]) if c["tree"] else None
        s["dout"] = _randn(g, B, L, T, H * c["G"], D).to(torch.bfloat16)
        s["out"], s["lse"] = _forward(s, c, s["store"])
        if c["pools"]:
            for x in ("dk_pool", "dv_pool"):
                s[x] = torch.zeros((units * per, PAGE, D), dtype=torch.bfloat16, device="cuda")
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program keeps between calls of the package: store, pages, outputs and workspace."""
    from paper_2608_21541_gb300 import certkv as ck
    c, t = s["case"], s["store"]
    if "k" not in t:  # the pages' operators do not touch the pool's rows
        t["k"] = t["v"] = torch.empty((t["pages"], PAGE, D), dtype=torch.bfloat16, device="cuda")
    s["handle"] = ck.Store(k=t["k"], v=t["v"], table=t["table"], counts=t["counts"],
                           format=t["format"], k_group=t.get("k_group"),
                           v_group=t.get("v_group"), k_scale=t.get("k_scale"),
                           v_scale=t.get("v_scale"))
    if c["op"] in ("list", "reserve"):
        s["pages"] = ck.Pages(held=s["held"], free=s["free"], free_count=s["n_free"])
        s["ws"] = ck.workspace(ck.certkv_pages_workspace_bytes(s["handle"]), "cuda")
    elif c["op"] == "map":
        s["slots"] = torch.empty((len(t["counts"]), c["T"]), dtype=torch.int32, device="cuda")
        s["positions"] = torch.empty((c["B"], c["T"]), dtype=torch.int32, device="cuda")
    else:
        s["dq"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["dk"] = torch.empty(s["k"].shape, dtype=torch.bfloat16, device="cuda")
        s["dv"] = torch.empty(s["v"].shape, dtype=torch.bfloat16, device="cuda")
        s["ws"] = ck.workspace(ck.certkv_tree_grad_workspace_bytes(
            c["B"], c["L"], c["H"] * c["G"], c["H"], c["T"]), "cuda")


# -------------------------------------------------------------------- run --
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2608_21541_gb300 import certkv as ck
    c, st = s["case"], s["handle"]
    if c["op"] == "list":
        ck.certkv_pages_list(st, s["pages"], ws=s["ws"])
        return _pages(s)
    if c["op"] == "reserve":
        ck.certkv_pages_reserve(st, s["pages"], s["no_room"], ws=s["ws"])
        ck.certkv_pages_reserve(st, s["pages"], s["rooms"], ws=s["ws"])
        return {"table": st.table, **_pages(s)}
    if c["op"] == "map":
        ck.certkv_slot_map(st, c["T"], rows=s["rows"], base=s["base"], mask=s["mask"],
                           slots=s["slots"], positions=s["positions"])
        return {"slots": s["slots"], "positions": s["positions"]}
    ck.certkv_tree_attn_grad(s["dout"], s["q"], st, s["out"], s["lse"], hkv=c["H"], k_new=s["k"],
                             v_new=s["v"], mask=s["mask"], dq=s["dq"], dk_new=s["dk"],
                             dv_new=s["dv"], dk_store=s.get("dk_pool"),
                             dv_store=s.get("dv_pool"), ws=s["ws"])
    return _grads(s, s["dq"], s["dk"], s["dv"])


def _pages(s):
    """held, and the pages that are free (what lies behind them in the list says nothing)."""
    n = torch.arange(len(s["free"]), device="cuda")
    return {"held": s["held"], "n_free": s["n_free"],
            "free": torch.where(n < s["n_free"], s["free"], -1)}


def _grads(s, dq, dk, dv):
    out = {"dq": dq, "dk": dk, "dv": dv}
    if s["case"]["pools"]:
        out["dk_pool"], out["dv_pool"] = s["dk_pool"], s["dv_pool"]
    return out


# ------------------------------------------------------- the plain forms --
def _run_plain(s):
    return {"list": _plain_list, "reserve": _plain_reserve, "map": _plain_map,
            "grad": _plain_grad}[s["case"]["op"]](s, s["case"], s["store"])


def _plain_list(s, c, t):
    table, pool = t["table"], t["pages"]
    owned = (table >= 0) & (table < pool)
    at = torch.arange(1, table.shape[1] + 1, device="cuda")
    s["held"].copy_((owned * at).amax(1))
    used = torch.zeros(pool + 1, dtype=torch.bool, device="cuda")
    used[torch.where(owned, table, pool).long()] = True
    free = ~used[:pool]
    n = free.sum()
    # the lowest page is the first to be handed out: it is the last of the list
    place = torch.where(free, n - torch.cumsum(free, 0), pool)
    ext = torch.full((pool + 1,), -1, dtype=torch.int32, device="cuda")
    ext[place] = torch.arange(pool, dtype=torch.int32, device="cuda")
    s["free"].copy_(ext[:pool])
    s["n_free"].copy_(n[None])
    return _pages(s)


def _plain_reserve(s, c, t):
    _plain_change(s, c, t, s["no_room"])
    _plain_change(s, c, t, s["rooms"])
    return {"table": t["table"], **_pages(s)}


def _plain_change(s, c, t, rooms):
    """Pages of every segment brought to what counts + rooms need."""
    table, held = t["table"], s["held"].long()
    units, most = table.shape
    want = torch.clamp(t["counts"] + rooms.repeat_interleave(c["L"] * c["H"], output_size=units),
                       min=0)
    need = torch.clamp((want.long() + PAGE - 1) // PAGE, max=most)
    t["counts"].copy_(torch.minimum(t["counts"], want))
    at = torch.arange(most, device="cuda")[None]
    gone = (at >= need[:, None]) & (at < held[:, None])
    more = (at >= held[:, None]) & (at < need[:, None])
    pool, n0 = t["pages"], s["n_free"].long()
    back = gone.sum()
    # the i-th page given back becomes entry n0 + back - 1 - i of the list
    i = torch.cumsum(gone.flatten(), 0).view_as(gone) - 1
    ext = torch.cat([s["free"], s["free"][:1]])
    ext[torch.where(gone, n0 + back - 1 - i, pool)] = table
    # the j-th page handed out is entry n0 + back - 1 - j
    j = torch.cumsum(more.flatten(), 0).view_as(more) - 1
    page = ext[torch.clamp(n0 + back - 1 - j, min=0)]
    table.copy_(torch.where(gone, -1, torch.where(more & (j < n0 + back), page, table)))
    got = (more & (j < n0 + back)).sum(1)
    s["held"].copy_(torch.where(need < held, need, held + got))
    s["free"].copy_(ext[:pool])
    s["n_free"].copy_(n0 + back - got.sum())


def _plain_map(s, c, t):
    B, T, units = c["B"], c["T"], c["B"] * c["L"] * c["H"]
    i = torch.arange(T, device="cuda")
    live = i[None] < s["rows"][:, None]
    idx = _slot(t["table"], t["counts"][:, None] + i[None])
    mine = live.repeat_interleave(units // B, 0, output_size=units)
    depth = i[None].expand(B, T)
    if s["mask"] is not None:
        bits = (s["mask"][..., None] >> i) & 1
        depth = bits.sum(-1) - torch.diagonal(bits, dim1=1, dim2=2)
    return {"slots": torch.where(mine, idx, -1).to(torch.int32),
            "positions": (s["base"][:, None] + depth).to(torch.int32)}


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


def _by_unit(x, c):
    """[B][L][T][H G][..] as [units][T G][..] in 32 bits."""
    U, G = c["B"] * c["L"] * c["H"], c["G"]
    x = x.unflatten(3, (c["H"], G)).movedim(3, 2)
    return x.reshape(U, c["T"] * G, *x.shape[5:]).float()


def _from_unit(x, c):
    """[units][T n][D] as bf16 [B][L][T][H n][D]."""
    B, L, T, H = c["B"], c["L"], c["T"], c["H"]
    return x.view(B, L, H, T, -1, D).movedim(2, 3).reshape(B, L, T, -1, D).to(torch.bfloat16)


def _logits(s, c, t):
    """q [U][T G][D], drafts' k, v [U][T][D], the pool slots [U][S], stored k, v [U][S][D], and
    the logits [U][T G][S + T], -inf where a row does not see."""
    B, L, H, G, T = c["B"], c["L"], c["H"], c["G"], c["T"]
    U, S = B * L * H, t["table"].shape[1] * PAGE
    q = _by_unit(s["q"], c)
    kn, vn = (s[x].transpose(2, 3).reshape(U, T, D).float() for x in ("k", "v"))
    at = torch.arange(S, device="cuda")[None].expand(U, S)
    idx = _slot(t["table"], at)
    k, v = _decode(t, "k", idx), _decode(t, "v", idx)
    x = torch.cat([q @ k.transpose(1, 2), q @ kn.transpose(1, 2)], -1) * (1.0 / math.sqrt(D))
    j = torch.arange(T, device="cuda")
    if s["mask"] is None:
        sees = (j[None, :] <= j[:, None])[None].expand(B, T, T)
    else:
        sees = (s["mask"][..., None] >> j) & 1 > 0
    sees = sees[:, None, :, None].expand(B, L * H, T, G, T).reshape(U, T * G, T)
    live = at < t["counts"][:, None]
    x = torch.where(torch.cat([live[:, None].expand(U, T * G, S), sees], -1), x, -math.inf)
    return q, kn, vn, idx, live, k, v, x


def _forward(s, c, t):
    """Attention's output (bf16) and log-sum-exp, as a forward pass leaves them."""
    B, L, H, G, T = c["B"], c["L"], c["H"], c["G"], c["T"]
    _, _, vn, idx, _, _, v, x = _logits(s, c, t)
    S = idx.shape[1]
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    l = p.sum(-1, keepdim=True)
    o = p[..., :S] @ v + p[..., S:] @ vn
    lse = (m + torch.log(l)).view(B, L, H, T, G).movedim(2, 3).reshape(B, L, T, H * G)
    return _from_unit(torch.where(l > 0, o / l, 0.0), c), lse.contiguous()


def _plain_grad(s, c, t):
    U, G, T = c["B"] * c["L"] * c["H"], c["G"], c["T"]
    scale = 1.0 / math.sqrt(D)
    q, kn, vn, idx, live, k, v, x = _logits(s, c, t)
    S = idx.shape[1]
    do, lse = _by_unit(s["dout"], c), _by_unit(s["lse"], c)[..., None]
    delta = (do * _by_unit(s["out"], c)).sum(-1, keepdim=True)
    p = torch.exp(x - torch.where(lse > -math.inf, lse, 0.0))
    dp = torch.cat([do @ v.transpose(1, 2), do @ vn.transpose(1, 2)], -1)
    ds = p * (dp - delta) * scale
    dq = ds[..., :S] @ k + ds[..., S:] @ kn
    dk = ds[..., S:].transpose(1, 2) @ q
    dv = p[..., S:].transpose(1, 2) @ do
    if c["pools"]:
        where = idx[live]
        for name, w, rows in (("dk_pool", ds, q), ("dv_pool", p, do)):
            new = w[..., :S].transpose(1, 2) @ rows
            s[name].view(-1, D)[where] = new[live].to(torch.bfloat16)
    return _grads(s, _from_unit(dq, c), _from_unit(dk, c), _from_unit(dv, c))


# ------------------------------------------------------------------- work --
ROW_BYTES = {"bf16": 2 * D, "fp8": D + 4, "fp4": D // 2 + D // 16 + 4}


def work(case):
    c = case
    units = c["B"] * c["L"] * c["H"]
    mean = c["slots"] * 15.0 / 16 if c.get("ragged", True) else c["slots"]
    if c["op"] == "list":
        pages = units * (1 + (mean + c["room"] / 2) / PAGE)
        return {"bytes": 4 * units + 4 * pages + 4 * pages / 8, "flops": 0}
    if c["op"] == "reserve":  # entries read and written twice over, in the table and in the list
        room = c["room"] if c["B"] == 1 else (c["room"] + 1) / 2
        return {"bytes": 2 * (12 * units + 4 * c["B"]) + 16 * units * room / PAGE, "flops": 0}
    if c["op"] == "map":
        rows = units * c["T"]
        read = (1 if c["ragged"] else 2) * rows / PAGE * 2 + 4 * units
        words = c["B"] * c["T"] * (12 if c["tree"] else 4)
        return {"bytes": 4 * rows + read + words, "flops": 0}
    rows, slots = units * c["G"] * c["T"], units * mean
    drafts = units * c["T"]
    more = 4 * D * slots if c["pools"] else 0
    return {"bytes": slots * 2 * ROW_BYTES[c["format"]] + rows * (8 * D + 4) + drafts * 8 * D + more,
            "flops": 2.0 * D * c["T"] * c["G"] * ((5 if c["pools"] else 3) * slots + 5 * drafts)}


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
    if case["op"] != "grad":
        return None
    s = prepare(case, seed)
    c, t = case, s["store"]
    L, H, G, T = c["L"], c["H"], c["G"], c["T"]
    got = {n: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda")
           for n, x in (("dq", "q"), ("dk", "k"), ("dv", "v"))}
    if c["pools"]:
        for x in ("dk_pool", "dv_pool"):
            got[x] = torch.zeros(s[x].shape, dtype=torch.float64, device="cuda")
    counts = t["counts"].cpu().tolist()
    words = None if s["mask"] is None else s["mask"].cpu().tolist()
    unseen = [torch.tensor([[j > i if words is None else not words[b][i] >> j & 1
                             for j in range(T)] for i in range(T)], device="cuda")
              for b in range(c["B"])]
    for u in range(c["B"] * L * H):
        b, l, h = u // (L * H), u // H % L, u % H
        n, heads = counts[u], slice(h * G, (h + 1) * G)
        at = torch.arange(n, device="cuda")
        slots = t["table"][u, at // PAGE].long() * PAGE + at % PAGE
        k = torch.cat([_held64(t, "k", slots), s["k"][b, l, :, h].double()])
        v = torch.cat([_held64(t, "v", slots), s["v"][b, l, :, h].double()])
        q, o, do = (s[x][b, l, :, heads].double().reshape(T * G, D) for x in ("q", "out", "dout"))
        lse = s["lse"][b, l, :, heads].double().reshape(T * G, 1)
        hide = torch.zeros((T, G, n + T), dtype=torch.bool, device="cuda")
        hide[:, :, n:] = unseen[b][:, None]
        prob = torch.exp(torch.addmm(-lse.expand(-1, n + T), q, k.T, alpha=1.0 / math.sqrt(D)))
        prob = prob.masked_fill(hide.view(T * G, -1), 0.0)
        pull = torch.einsum("rd,sd->rs", do, v) - torch.einsum("rd,rd->r", do, o)[:, None]
        flow = prob * pull / math.sqrt(D)
        got["dq"][b, l, :, heads] = (flow @ k).view(T, G, D)
        dk, dv = flow.T @ q, prob.T @ do
        got["dk"][b, l, :, h], got["dv"][b, l, :, h] = dk[n:], dv[n:]
        if c["pools"]:
            got["dk_pool"].view(-1, D)[slots] = dk[:n]
            got["dv_pool"].view(-1, D)[slots] = dv[:n]
    return got
