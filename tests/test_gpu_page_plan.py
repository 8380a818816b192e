"""pbd_page_plan and pbd_page_release against a plain allocator: who is served, which pages in which order, rows and slots,
and what a bad stack, table or length leaves as it was."""
import copy
import random

import pytest
import torch

import rows_ref as rr
from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def make(rng, B, W, page, pages, most):
    """A pool of which some pages are with sequences, some free, some with others."""
    ids = list(range(pages))
    rng.shuffle(ids)
    have = [rng.randint(0, min(W, most)) for _ in range(B)]
    table = [[ids.pop() if p < h else -1 for p in range(W)] for h in have]
    n = rng.randint(0, len(ids))
    free = ids[:n] + [-1] * (pages - n)
    return rr.Tables(table, have, free, n, page)


class Pool:
    def __init__(self, t):
        self.t = t
        self.table, self.seq_pages, self.free, self.n_free = i32(t.table), i32(t.seq_pages), i32(t.free), i32([t.n_free])
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def plan(self, lens, new, pos, R, plain=False):
        B = len(lens)
        o = {n: torch.full((s,), -55, dtype=torch.int32, device=DEV)
             for n, s in (("row_start", B + 1), ("row_seq", R), ("row_pos", R), ("slot_map", R), ("new_lens", B))}
        self.status.zero_()
        pbd.pbd_page_plan(self.table, self.seq_pages, self.free, self.n_free, i32(lens), i32(new), self.t.page, o["row_start"],
                          None if plain else o["row_seq"], o["slot_map"], o["new_lens"], pos=None if plain else i32(pos),
                          row_pos=None if plain else o["row_pos"], status=self.status)
        return {n: v.tolist() for n, v in o.items()}

    def release(self, keep):
        self.status.zero_()
        pbd.pbd_page_release(self.table, self.seq_pages, self.free, self.n_free, i32(keep), self.t.page, status=self.status)

    def same(self):
        t = self.t
        assert self.table.tolist() == t.table
        assert self.seq_pages.tolist() == t.seq_pages
        assert self.n_free.tolist() == [t.n_free]
        assert self.free.tolist()[: max(0, t.n_free)] == t.free[: max(0, t.n_free)]

    def check_plan(self, lens, new, pos, R):
        got = self.plan(lens, new, pos, R)
        want = self.t.plan(lens, new, pos, R)
        assert int(self.status) == want.pop("status")
        for n, v in want.items():
            assert got[n] == v, n
        self.same()
        return got


@pytest.mark.parametrize("seed", range(12))
def test_plans_and_releases(seed):
    """Random pools, demands that fit and that do not, rows by one work-group (below 4097) and by many."""
    rng = random.Random(seed)
    B = [1, 2, 7, 64, 65, 200, 1024, 1025, 2500, 3, 33, 300][seed]
    page = rng.choice([16, 32, 128, 4096])
    W = rng.randint(1, 9)
    t = make(rng, B, W, page, B * W + 5, 5)
    p = Pool(t)
    for _ in range(3):
        lens = [rng.randint(0, h * page) for h in t.seq_pages]
        room = [W * page - m for m in lens]
        new = [rng.choice([0, 0, 1, rng.randint(0, r), rng.randint(0, min(r, 40))]) for r in room]
        if seed % 3 == 0:
            new = [min(n, 3) for n in new]
        R = sum(new) + rng.choice([0, 1, 70])
        if R > 300000:
            new = [min(n, 90) for n in new]
            R = sum(new)
        pos = [rng.randint(0, 1000) for _ in lens]
        got = p.check_plan(lens, new, pos, R)
        keep = [rng.choice([m, m, 0, rng.randint(0, W * page + 3)]) for m in got["new_lens"]]
        p.release(keep)
        assert t.release(keep) == int(p.status) == 0
        p.same()


def test_a_release_undoes_a_plan():
    rng = random.Random(5)
    t = make(rng, 20, 12, 16, 400, 3)
    t.free = t.free[: t.n_free] + [-1] * (400 - t.n_free)
    p = Pool(t)
    before = copy.deepcopy(t.__dict__)
    lens = [h * 16 for h in t.seq_pages]
    p.plan(lens, [rng.randint(0, 100) for _ in lens], lens, 4000)
    p.release(lens)
    t.__dict__ = before
    p.same()


def test_rows_past_the_bound():
    t = rr.Tables([[-1] * 4 for _ in range(3)], [0] * 3, list(range(20)), 20, 16)
    p = Pool(t)
    p.check_plan([0, 0, 0], [10, 30, 5], [0, 7, 9], 38)
    assert int(p.status) == 1
    p.check_plan([10, 0, 0], [0, 0, 0], [0, 7, 9], 0)


@pytest.mark.parametrize("many", [False, True])
def test_without_positions_and_sequences(many):
    n = 3000 if many else 30
    t = rr.Tables([[-1] * 400 for _ in range(2)], [0] * 2, list(range(900)), 900, 16)
    p = Pool(t)
    got = p.plan([0, 0], [n, n], None, 2 * n + 2, plain=True)
    want = t.plan([0, 0], [n, n], [0, 0], 2 * n + 2)
    assert got["slot_map"] == want["slot_map"] and got["row_start"] == want["row_start"]
    assert got["row_seq"] == [-55] * (2 * n + 2)
    p.same()


def test_bad_lengths_skip_the_sequence():
    """Out of range by the sign, by the table, by the pages that it has; sums past 31 bits."""
    big = 2 ** 31 - 1
    t = rr.Tables([[1, -1], [2, -1], [3, -1], [4, -1], [5, -1], [6, -1]], [1, 1, 1, 1, 3, -1], list(range(20)), 20, 16)
    p = Pool(t)
    p.check_plan([16, -1, 16, 17, 5, 0], [16, 3, -2, 1, 1, 1], [0] * 6, 100)
    p.check_plan([16, 16, 16, 16, 0, 0], [big, big, big, big, 0, 0], [0] * 6, 100)
    p.check_plan([big, 16, 16, 16, 0, 0], [1, 1, 1, 1, 0, 0], [0] * 6, 100)


def test_bad_stacks_serve_nobody_who_needs_a_page():
    for n_free in (-1, 9, 2 ** 31 - 1, -2 ** 31):
        t = rr.Tables([[0, -1], [1, -1]], [1, 1], [2, 3, 4, 5, 6, 7, 8, 0], n_free, 16)
        t2 = copy.deepcopy(t)
        t2.free = t.free[:]
        p = Pool(t)
        got = p.plan([3, 16], [4, 4], [0, 0], 10)
        assert got["new_lens"] == [7, 16] and int(p.status) == 1 and p.n_free.tolist() == [n_free]
        assert got["slot_map"] == [3, 4, 5, 6, -1, -1, -1, -1, -1, -1]
        p.release([0, 0])
        assert int(p.status) == 1 and p.table.tolist() == t2.table and p.seq_pages.tolist() == [1, 1]
    for bad in (-1, 8, 2 ** 31 - 1):
        t = rr.Tables([[0, -1], [1, -1]], [1, 1], [2, 3, bad, 5, -1, -1, -1, -1], 3, 16)
        p = Pool(t)
        p.check_plan([3, 16], [4, 4], [0, 0], 10)
        assert int(p.status) == 17


def test_bad_tables_keep_their_pages():
    t = rr.Tables([[0, 1, 9], [2, 3, -1], [4, 5, 6], [7, -1, -1]], [3, 3, 3, 4], [-1] * 9, 0, 16)
    p = Pool(t)
    keep = [16, 16, 20, 0]
    p.release(keep)
    assert t.release(keep) == int(p.status) == 17
    p.same()
    p.release([-1, 48, 17, 0])
    assert int(p.status) & 1
    # more pages than the stack has room for
    t = rr.Tables([[0, 1], [2, 3]], [2, 2], [0, 1, 2, -1], 3, 16)
    p = Pool(t)
    p.release([0, 0])
    assert t.release([0, 0]) == int(p.status) == 1
    p.same()


def test_captured_and_replayed():
    """A plan and its release as a graph, replayed with other lengths in the same tensors."""
    rng = random.Random(3)
    t = make(rng, 9, 20, 16, 300, 2)
    t.n_free = len([x for x in t.free if x >= 0])
    p = Pool(t)
    lens, new = i32([0] * 9), i32([0] * 9)
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (10, 400, 400, 9)]

    def call():
        pbd.pbd_page_plan(p.table, p.seq_pages, p.free, p.n_free, lens, new, 16, out[0], out[1], out[2], out[3], status=p.status)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    at = [min(5, 16 * h) for h in t.seq_pages]
    for _ in range(3):
        add = [rng.randint(0, 40) for _ in range(9)]
        lens.copy_(i32(at))
        new.copy_(i32(add))
        graph.replay()
        want = t.plan(at, add, [0] * 9, 400)
        torch.cuda.synchronize()
        assert [out[i].tolist() for i in range(4)] == [want[n] for n in ("row_start", "row_seq", "slot_map", "new_lens")]
        p.same()
        at = want["new_lens"]
