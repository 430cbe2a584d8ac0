"""Verifying drafted tokens over a compressed, quantised KV cache.

A prefilled cache is compressed to its exact budget and quantised into a paged
store; then every step drafts a tree of tokens, rotates their queries and keys,
attends them over the store and over each other, and appends the accepted path's
keys and values to the store.  The model around the attention is replaced by
seeded random projections, so the acceptance is random too.

    python examples/verify_drafts.py [--format fp8] [--steps 16] [--tokens 16]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_21541_gb300 import certkv as ck  # noqa: E402
from paper_2608_21541_gb300 import workloads as W  # noqa: E402


def draft_tree(T: int, rng: torch.Generator):
    """(parents, words): a random tree over T drafts (parent -1: the committed text) and the
    drafts each token sees, itself and its ancestors, as bits of an int64 word."""
    pick = torch.rand(T, generator=rng).tolist()
    parents = [min(i - 1, int(pick[i] * (i + 1)) - 1) for i in range(T)]
    words = []
    for i, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << i)
    return parents, [w - (1 << 64) if w >> 63 else w for w in words]


def accepted_path(parents, leaf: int):
    path = []
    while leaf >= 0:
        path.append(leaf)
        leaf = parents[leaf]
    return path[::-1]


def run(wl: W.Workload, fmt: str = "fp8", steps: int = 16, T: int = 16, seed: int = 0,
        on_step=None) -> dict:
    """Compress, store and verify `steps` trees of T drafts; on_step(step, q, k, v, mask, out,
    store) sees every step's rotated inputs and output before the store grows."""
    dev = torch.device("cuda")
    rng = torch.Generator().manual_seed(seed)
    K, V, Q = W.draw(wl, seed=seed, device=dev)
    packed = ck.certkv_compress(K, V, Q, wl.B_live)
    del K, V

    # room for every accepted token; pages are handed out by the load
    room = steps * T
    longest = int(packed.real_counts.max().item()) + 1 + room
    total = wl.B * wl.L * wl.B_live
    store = ck.Store.empty(wl.units, -(-longest // ck.STORE_PAGE), fmt,
                           pool_pages=(total + wl.units * room) // ck.STORE_PAGE + 2 * wl.units,
                           device=dev)
    ck.certkv_store_load(packed, store, room)

    plan = ck.certkv_rope_plan(wl.d)
    shape = (wl.B, wl.L, T)
    out = torch.empty((*shape, wl.Hq, wl.d), dtype=torch.bfloat16, device=dev)
    ws = ck.workspace(ck.certkv_tree_workspace_bytes(wl.B, wl.L, wl.Hq, wl.H, T), dev)
    length = wl.n  # position of the next token: the compressed context keeps its own
    grown, spent = 0, 0.0
    for step in range(steps):
        trees = [draft_tree(T, rng) for _ in range(wl.B)]
        mask = torch.tensor([w for _, w in trees], device=dev)
        depth = [[len(accepted_path(p, i)) - 1 for i in range(T)] for p, _ in trees]
        positions = torch.tensor(depth, dtype=torch.int32, device=dev) + length
        g = torch.Generator(device=dev).manual_seed(seed * 1000 + step)
        qkv = torch.randn((*shape, wl.Hq + 2 * wl.H, wl.d), generator=g, device=dev).to(
            torch.bfloat16)
        q, k, v = qkv.split((wl.Hq, wl.H, wl.H), dim=3)  # views: no copies below
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        ck.certkv_rope(q, positions, plan, k, out=q, k_out=k)
        ck.certkv_tree_attn(q, store, hkv=wl.H, k_new=k, v_new=v, mask=mask, out=out, ws=ws)
        if on_step is not None:
            on_step(step, q, k, v, mask, out, store)
        # one path of every tree is accepted
        leaves = [int(torch.randint(0, T, (1,), generator=rng)) for _ in range(wl.B)]
        paths = [accepted_path(p, leaf) for (p, _), leaf in zip(trees, leaves)]
        n = min(len(p) for p in paths)  # one length for all sequences keeps positions simple
        select = torch.tensor([p[:n] + [0] * (T - n) for p in paths], dtype=torch.int32,
                              device=dev)
        accepted = torch.full((wl.B,), n, dtype=torch.int32, device=dev)
        ck.certkv_store_append(k, v, store, select=select, accepted=accepted)
        torch.cuda.synchronize()
        spent += time.perf_counter() - t0
        length += n
        grown += n
    return dict(store=store, packed=packed, accepted=grown, ms_per_step=spent / steps * 1e3)


def main():
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--format", choices=tuple(ck.STORE_FORMATS), default="fp8")
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--context", type=int, default=32768)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    wl = W.WORKLOADS["C2"].with_(n=a.context, L=a.layers)
    r = run(wl, a.format, a.steps, a.tokens)
    kept = r["store"].counts.sum().item()
    print(f"{wl.L} layers x {wl.H} KV heads x {wl.n} tokens compressed to {wl.B_live} slots a "
          f"layer, stored as {a.format}; {r['accepted']} of {a.steps * a.tokens} drafts accepted, "
          f"{kept} slots live, {r['ms_per_step']:.3f} ms a step, status {r['store'].read_status()}")


if __name__ == "__main__":
    main()
