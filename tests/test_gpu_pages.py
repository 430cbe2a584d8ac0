"""A store's pages kept on the GPU: free list, reservation and slot map, against a plain
restatement of include/certkv.h in Python integers.  Everything is a whole number: equality."""
import numpy as np
import pytest
import torch

import drafts
from paper_2608_21541_gb300 import certkv as ck

pytestmark = pytest.mark.gpu
PAGE = drafts.PAGE


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def store(units, max_pages, pool, table=None, counts=None):
    """A store whose rows nobody looks at: a small pool repeated is not needed, 4-bit is small."""
    st = ck.Store.empty(units, max_pages, "fp4", pool_pages=pool)
    if table is not None:
        st.table.copy_(ints(table))
    if counts is not None:
        st.counts.copy_(ints(counts))
    return st


class Account:
    """The definition, on the host."""

    def __init__(self, st, pg=None):
        self.table, self.counts = st.table.cpu().numpy().copy(), st.counts.cpu().numpy().copy()
        self.pool = st.k.shape[0]
        self.status = 0
        if pg is not None:
            n = int(pg.free_count[0])
            self.held, self.free = pg.held.cpu().numpy().copy(), list(pg.free[:n].cpu().numpy())

    def list(self):
        page = (self.table >= 0) & (self.table < self.pool)
        self.held = np.array([max([i + 1 for i in np.flatnonzero(r)], default=0) for r in page])
        used = set(self.table[page].tolist())
        self.free = [p for p in range(self.pool - 1, -1, -1) if p not in used]

    def reserve(self, room, want=None, batch=1):
        U, most = self.table.shape
        per = U // batch
        base = self.counts if want is None else want
        s = [int(base[u]) + (int(room[u // per]) if room is not None else 0) for u in range(U)]
        if any(x > most * PAGE for x in s):
            self.status = ck.STATUS_STORE
        s = [min(max(x, 0), most * PAGE) for x in s]
        need = [-(-x // PAGE) for x in s]
        back = []
        for u in range(U):
            back += self.table[u, need[u]:self.held[u]].tolist()
            self.table[u, need[u]:max(need[u], self.held[u])] = -1
        room_left = self.pool - len(self.free)
        if len(back) > room_left:
            self.status = ck.STATUS_STORE
        self.free += back[:room_left][::-1]
        for u in range(U):
            have = min(self.held[u], need[u])
            while have < need[u] and self.free:
                page = self.free.pop()
                self.table[u, have] = page
                have += 1
                if not 0 <= page < self.pool:
                    self.status = ck.STATUS_STORE
            if have < need[u]:
                self.status = ck.STATUS_STORE
            self.held[u] = have
            self.counts[u] = min(self.counts[u], s[u])

    def check(self, st, pg):
        np.testing.assert_array_equal(pg.held.cpu().numpy(), self.held)
        assert int(pg.free_count[0]) == len(self.free)
        np.testing.assert_array_equal(pg.free[:len(self.free)].cpu().numpy(), self.free)
        np.testing.assert_array_equal(st.table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(st.counts.cpu().numpy(), self.counts)
        assert st.read_status() == self.status


def random_store(units, max_pages, pool, seed, share=0.5):
    """Segments of 0 .. max_pages pages, their pages in no order."""
    rng = np.random.default_rng(seed)
    held = rng.integers(0, max_pages + 1, units)
    while held.sum() > share * pool:
        held = held // 2
    order = rng.permutation(pool)
    table = np.full((units, max_pages), -1)
    at = 0
    for u in range(units):
        table[u, :held[u]] = order[at:at + held[u]]
        at += held[u]
    counts = np.minimum(rng.integers(0, PAGE, units) + (held - 1) * PAGE + 1, held * PAGE)
    return store(units, max_pages, pool, table, np.maximum(counts, 0)), rng


SHAPES = [(1, 1, 1), (3, 5, 11), (64, 16, 700), (1000, 3, 1601), (257, 300, 50000), (5000, 8, 30011),
          (20000, 2, 32769)]


@pytest.mark.parametrize("units,max_pages,pool", SHAPES)
def test_list(units, max_pages, pool):
    st, _ = random_store(units, max_pages, pool, units)
    pg = ck.certkv_pages_list(st)
    a = Account(st)
    a.list()
    a.check(st, pg)


def test_list_of_rows_with_holes_and_foreign_entries():
    table = [[5, -1, 3, -1], [-1, -1, -1, -1], [9, 1 << 30, -7, 0], [40, -1, -1, -1]]
    st = store(4, 4, 10, table)
    pg = ck.certkv_pages_list(st)
    assert pg.held.tolist() == [3, 0, 4, 0]
    assert pg.free[:int(pg.free_count[0])].tolist() == [8, 7, 6, 4, 2, 1]


@pytest.mark.parametrize("pool", [1, 31, 32, 33, 32767, 32768, 32769, 100001])
def test_list_of_an_empty_store(pool):
    st = store(2, 3, pool)
    pg = ck.certkv_pages_list(st)
    assert int(pg.free_count[0]) == pool
    assert torch.equal(pg.free.cpu(), torch.arange(pool - 1, -1, -1, dtype=torch.int32))


@pytest.mark.parametrize("units,max_pages,pool", SHAPES)
@pytest.mark.parametrize("batch", ["one", "many"])
def test_reserve_over_steps(units, max_pages, pool, batch):
    """Lengths that grow, shrink and end, pools that run out among them."""
    st, rng = random_store(units, max_pages, pool, 7 * units)
    B = 1 if batch == "one" else max(d for d in (1, 2, 3, 8, 1000, 5000) if units % d == 0)
    pg = ck.certkv_pages_list(st)
    a = Account(st)
    a.list()
    ws = ck.workspace(ck.certkv_pages_workspace_bytes(st), "cuda")
    for step in range(6):
        room = rng.integers(-2 * PAGE, 3 * PAGE, B)
        room[rng.random(B) < 0.2] = -2 ** 31
        want = None
        if step % 2:
            want = rng.integers(0, max_pages * PAGE + 1, units)
        ck.certkv_pages_reserve(st, pg, ints(room), want=None if want is None else ints(want), ws=ws)
        a.reserve(room, want, B)
        a.check(st, pg)
        grown = np.minimum(a.counts + rng.integers(0, PAGE, units), a.held * PAGE)
        a.counts = grown.astype(a.counts.dtype)
        st.counts.copy_(ints(grown))


def test_what_is_taken_back_restores_the_list():
    st, rng = random_store(300, 40, 20000, 5)
    pg = ck.certkv_pages_list(st)
    before = [x.clone() for x in (st.table, pg.held, pg.free_count)]
    free = pg.free[:int(pg.free_count[0])].clone()
    for n in (1, 64, 1000):
        ck.certkv_pages_reserve(st, pg, ints([n]))
        assert int(pg.free_count[0]) < len(free)
        ck.certkv_pages_reserve(st, pg, ints([0]))
        assert all(torch.equal(x, y) for x, y in zip(before, (st.table, pg.held, pg.free_count)))
        assert torch.equal(pg.free[:len(free)], free)


def test_reserve_refuses_nothing_it_can_answer():
    """Accounts out of range, and lengths past a row: clamped, never followed."""
    st = store(4, 3, 8, [[0, 1, -1], [2, -1, -1], [3, 4, 5], [-1, -1, -1]], [100, 7, 150, 0])
    pg = ck.Pages(held=ints([2, 1, 3, 0]), free=ints([6, 99, 7, 0, 0, 0, 0, 0]),
                  free_count=ints([3]))
    a = Account(st, pg)
    ck.certkv_pages_reserve(st, pg, ints([50]))
    a.reserve([50])
    a.check(st, pg)
    assert st.read_status() == ck.STATUS_STORE
    # a count above the pool and a negative held are read as clamped
    st2 = store(2, 3, 4, [[0, 1, 2], [3, -1, -1]], [10, 5])
    pg2 = ck.Pages(held=ints([100, -5]), free=ints([0, 0, 0, 0]), free_count=ints([77]))
    ck.certkv_pages_reserve(st2, pg2, None, want=ints([0, 0]))
    assert pg2.held.tolist() == [0, 0] and int(pg2.free_count[0]) == 4
    assert st2.counts.tolist() == [0, 0] and st2.read_status() == ck.STATUS_STORE


def test_want_alone_and_neither():
    st, _ = random_store(24, 9, 150, 3)
    pg = ck.certkv_pages_list(st)
    a = Account(st, pg)
    ck.certkv_pages_reserve(st, pg)  # down to the live slots
    a.reserve(None)
    a.check(st, pg)
    want = np.arange(24) * 20
    ck.certkv_pages_reserve(st, pg, want=ints(want), batch=8)
    a.reserve(None, want)
    a.check(st, pg)


def map_of(st, T, rows=None, start=None, base=None, mask=None, batch=1):
    table, counts = st.table.cpu().numpy().astype(np.int64), st.counts.cpu().numpy()
    U, most = table.shape
    per = U // batch
    slots = np.full((U, T), -1, np.int64)
    for u in range(U):
        n = T if rows is None else min(max(int(rows[u // per]), 0), T)
        s = np.arange(n) + (int(counts[u]) if start is None else int(start[u]))
        ok = (s >= 0) & (s < most * PAGE)
        page = table[u, np.where(ok, s, 0) // PAGE]
        ok &= (page >= 0) & (page < st.k.shape[0])
        slots[u, :n] = np.where(ok, page * PAGE + s % PAGE, -1)
    pos = np.zeros((batch, T), np.int64)
    for b in range(batch):
        for t in range(T):
            depth = t
            if mask is not None:
                w = int(mask[b][t])
                depth = sum(w >> j & 1 for j in range(T) if j != t)
            pos[b, t] = (0 if base is None else int(base[b])) + depth
    return slots, pos


@pytest.mark.parametrize("units,batch,T", [(1, 1, 1), (6, 3, 7), (64, 8, 64), (10, 2, 129), (3, 1, 5000),
                                           (2000, 1000, 33)])
@pytest.mark.parametrize("given", [False, True])
def test_slot_map(units, batch, T, given):
    max_pages = 3 + T // PAGE
    st, rng = random_store(units, max_pages, 2 * units * max_pages, T + units, share=1.0)
    rows = rng.integers(-1, T + 3, batch) if given else None
    start = rng.integers(-5, max_pages * PAGE, units) if given else None
    base = rng.integers(0, 2 ** 30, batch) if given else None
    mask = None
    if T <= 64 and given:
        mask = np.array([drafts.random_tree(T, rng) for _ in range(batch)])
        if T < 64:
            mask |= -1 << T  # bits past the tokens
        mask[0, T // 2] = 0
    got = ck.certkv_slot_map(st, T, rows=None if rows is None else ints(rows),
                             start=None if start is None else ints(start),
                             base=None if base is None else ints(base),
                             mask=None if mask is None else torch.tensor(mask).cuda(), batch=batch)
    want = map_of(st, T, rows, start, base, mask, batch)
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x.cpu().numpy(), y)


def test_positions_wrap_and_outputs_may_be_left_out():
    st, _ = random_store(4, 2, 20, 1)
    L, s = ck.load_library(), st.struct()
    import ctypes
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    base = ints([2 ** 31 - 2, -5])
    assert L.certkv_slot_map(2, 3, None, None, base.data_ptr(), None, ctypes.byref(s), None,
                             pos.data_ptr(), None) == ck.OK
    torch.cuda.synchronize()
    assert pos.tolist() == [[2 ** 31 - 2, 2 ** 31 - 1, -2 ** 31], [-5, -4, -3]]


def test_a_step_in_a_graph_on_another_stream():
    """Reserve, map, append and attend captured together: every replay goes on from what the
    one before left, and the map names the slots that the append fills."""
    B, L, H, T = 2, 1, 2, 5
    st = ck.Store.empty(B * L * H, 6, "bf16", pool_pages=40)
    pg = ck.certkv_pages_list(st)
    ws = ck.workspace(ck.certkv_pages_workspace_bytes(st), "cuda")
    k, v = (drafts.randn((B, L, T, H, 128), i) for i in (1, 2))
    room = ints([T, T])
    slots = torch.empty((B * L * H, T), dtype=torch.int32, device="cuda")
    pos = torch.empty((B, T), dtype=torch.int32, device="cuda")
    base = torch.zeros(B, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ck.certkv_pages_reserve(st, pg, room, ws=ws)
        ck.certkv_slot_map(st, T, base=base, slots=slots, positions=pos)
        ck.certkv_store_append(k, v, st)
        base.add_(T)
    for step in range(60):
        graph.replay()
        torch.cuda.synchronize()
        count = (step + 1) * T
        assert st.counts.tolist() == [count] * 4 and st.read_status() == 0
        assert pg.held.tolist() == [-(-count // PAGE)] * 4
        assert pos.tolist() == [[step * T + i for i in range(T)]] * 2
        rows = st.k.view(-1, 128)[slots.long()]
        assert torch.equal(rows, k.permute(0, 1, 3, 2, 4).reshape(4, T, 128))
    owned = st.table[st.table >= 0].tolist()
    assert len(set(owned)) == len(owned) == 20
    assert sorted(owned + pg.free[:int(pg.free_count[0])].tolist()) == list(range(40))
