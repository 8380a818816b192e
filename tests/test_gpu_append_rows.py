"""pbd_paged_append_rows against a plain form in 64 bits: rows in any order over blocks and pages, types, norms, strides,
rows that are skipped, and what must stay as it was."""
import math

import pytest
import torch

import paged_ref as ref
from paper_2607_12422_amd import binding as pbd
from test_gpu_paged_append import half_step, rope_table, rotated

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


class Call:
    """Rows for the slots lens[b] .. of sequences (row r: (sequence, slot) of `where`, None: skipped)."""

    def __init__(self, where, lens, room, H, G, D, dtype, page=16, major="page", norm=True, with_q=True, pad=0, seed=0, pos=None):
        g = torch.Generator().manual_seed(seed)
        HQ, R = H * G, len(where)
        self.c = ref.Cache(lens, H, D, dtype, page=page, major=major, seed=seed, room=room)
        self.where, self.R, self.H, self.HQ, self.D, self.dtype = where, R, H, HQ, D, dtype
        x = torch.randn(R, (HQ + 2 * H) * D + pad, generator=g) * 3
        for r, w in enumerate(where):
            if w is None:
                x[r] = math.nan
        self.q, self.k, self.v = x[:, : HQ * D], x[:, HQ * D: (HQ + H) * D], x[:, (HQ + H) * D: (HQ + 2 * H) * D]
        dx = x.to(DEV)
        self.dq, self.dk, self.dv = dx[:, : HQ * D], dx[:, HQ * D: (HQ + H) * D], dx[:, (HQ + H) * D: (HQ + 2 * H) * D]
        if not with_q:
            self.dq = None
        self.gains = [(1 + 0.1 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in range(2)]
        self.pos = pos if pos is not None else [3 if w is None else w[1] // 2 + 5 for w in where]
        self.rope = rope_table(max(self.pos, default=0) + 1, D)
        t = self.c.table
        self.slots = [-1 - r % 3 if w is None else int(t[w[0], w[1] // page]) * page + w[1] % page for r, w in enumerate(where)]
        k, v, table = self.c.to(DEV)
        self.k0, self.v0, self.pool = k.clone(), v.clone(), (k, v)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.pages = pbd.make_pages(k, v, table, n_q_heads=HQ, head_dim=D, status=self.status)
        self.q_out = torch.full((R, HQ * D), 77.0, dtype=dtype, device=DEV) if with_q else None

    def run(self, **kw):
        dev = [None if t is None else t.to(DEV) for t in self.gains]
        i = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
        pbd.pbd_paged_append_rows(self.pages, self.dk, self.dv, i(self.slots), i(self.pos), self.rope.to(DEV), q=self.dq,
                                  q_out=self.q_out, q_norm=dev[0] if self.dq is not None else None, k_norm=dev[1], **kw)
        torch.cuda.synchronize()

    def check(self):
        k, v = (t.cpu() for t in self.pool)
        wk, wv = self.k0.cpu().clone(), self.v0.cpu().clone()
        live = [r for r, w in enumerate(self.where) if w is not None]
        if live:
            at = self.rope[[self.pos[r] for r in live]]
            want, tol = rotated(self.k[live].unflatten(1, (self.H, self.D)), self.gains[1], at, 1e-6)
            value = self.v[live].unflatten(1, (self.H, self.D))
            for b in range(len(self.c.lens)):
                mine = [i for i, r in enumerate(live) if self.where[r][0] == b]
                if not mine:
                    continue
                page, ik, iv = self.c.places(b, torch.tensor([self.where[live[i]][1] for i in mine]))
                for h in range(self.H):
                    got, w = k[page[:, None], h, ik].double(), want[mine, h]
                    assert torch.all((got - w).abs() <= tol[mine, h] + half_step(w, self.dtype) * 1.01)
                    assert torch.equal(v[page[:, None], h, iv], value[mine, h].to(self.dtype))
                    wk[page[:, None], h, ik] = k[page[:, None], h, ik]
                    wv[page[:, None], h, iv] = v[page[:, None], h, iv]
            if self.q_out is not None:
                wq, tq = rotated(self.q[live].unflatten(1, (self.HQ, self.D)), self.gains[0], at, 1e-6)
                got = self.q_out.double().cpu().unflatten(1, (self.HQ, self.D))[live]
                assert torch.all((got - wq).abs() <= tq + half_step(wq, self.dtype) * 1.01)
        if self.q_out is not None:
            dead = [r for r in range(self.R) if self.where[r] is None]
            assert torch.all(self.q_out[dead] == 77.0)
        same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
        assert same(k, wk) and same(v, wv)


def runs(lens, counts):
    return [(b, m + i) for b, (m, n) in enumerate(zip(lens, counts)) for i in range(n)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,counts", [([0], [1]), ([5, 16, 33], [17, 1, 30]), ([3, 0, 14, 100], [0, 300, 333, 16]),
                                         ([1, 2, 3, 7], [200, 201, 202, 203])])
def test_rows_of_sequences(lens, counts, dtype, D):
    for norm in (True, False):
        c = Call(runs(lens, counts), lens, max(counts), 2, 2, D, dtype, norm=norm, seed=D)
        c.run()
        c.check()
        assert int(c.status) == 0


@pytest.mark.parametrize("H,G,n", [(1, 1, 700), (3, 3, 400), (5, 1, 300), (8, 2, 100), (8, 4, 90), (1, 40, 300)])
def test_heads_with_and_without_queries(H, G, n):
    for with_q in (True, False):
        c = Call(runs([9, 2], [n, 7]), [9, 2], n, H, G, 128, BF, with_q=with_q, pad=8, seed=G)
        c.run()
        c.check()


@pytest.mark.parametrize("page", [16, 64, 4096])
@pytest.mark.parametrize("major", ["page", "head"])
def test_pages_and_strides(page, major):
    c = Call(runs([30, 0, 15], [150, 77, 400]), [30, 0, 15], 400, 3, 2, 64, BF, page=page, major=major, seed=page)
    c.run()
    c.check()


@pytest.mark.parametrize("n", [40, 900])
def test_rows_in_any_order_and_rows_that_are_skipped(n):
    g = torch.Generator().manual_seed(n)
    where = runs([7, 90, 0], [n, 5, n // 2])
    mixed = [where[i] for i in torch.randperm(len(where), generator=g)]
    for order in (mixed, where[::-1], [w if i % 3 else None for i, w in enumerate(where)], [None] * 30 + where + [None] * 17,
                  [None] * n):
        c = Call(order, [7, 90, 0], n, 2, 2, 128, BF, seed=n, pos=[(7 * i) % 50 for i in range(len(order))])
        c.run()
        c.check()
        assert int(c.status) == 0


@pytest.mark.parametrize("n", [20, 900])
def test_slots_and_positions_out_of_range_are_skipped(n):
    lens = [4]
    c = Call(runs(lens, [n]), lens, n, 2, 2, 64, BF, seed=n)
    last = c.pool[0].shape[0] * 16
    good = list(c.slots)
    for bad in (last, 2 ** 31 - 1):
        c.slots[3] = bad
        c.where[3] = None
        c.status.zero_()
        c.run()
        c.check()
        assert int(c.status) == pbd.PBD_STATUS_PAGE
    c = Call(runs(lens, [n]), lens, n, 2, 2, 64, BF, seed=n)
    assert c.slots == good
    for bad in (-1, len(c.rope), 2 ** 31 - 1):
        pos = list(c.pos)
        c.pos[5] = bad
        c.where[5] = None
        c.status.zero_()
        c.run()
        c.pos = pos
        c.check()
        assert int(c.status) == pbd.PBD_STATUS_CAPACITY


def test_no_rows():
    c = Call([], [4], 4, 2, 2, 64, BF)
    c.run()
    c.check()


def test_offsets_past_32_bits():
    H, D, page, n = 8, 128, 64, 2 ** 31 // (8 * 128 * 64) + 40
    k, v = (torch.zeros(n, H, page * D, dtype=BF, device=DEV) for _ in range(2))
    pages = pbd.make_pages(k, v, torch.zeros(1, 1, dtype=torch.int32, device=DEV), n_q_heads=H, head_dim=D)
    g = torch.Generator().manual_seed(3)
    for R in (8, 800):
        x = torch.randn(R, H * D, generator=g)
        slots = torch.arange((n - 20) * page, (n - 20) * page + R, dtype=torch.int32)
        rope = rope_table(1, D)
        pbd.pbd_paged_append_rows(pages, x.to(DEV), x.to(DEV), slots.to(DEV), torch.zeros(R, dtype=torch.int32, device=DEV),
                                  rope.to(DEV))
        got_k, got_v = (t[n - 20:].cpu().unflatten(2, (4, 16 * D)) for t in (k, v))
        mk, mv = ref.block_maps(D, 8)
        s = torch.arange(R)
        want = x.to(BF).unflatten(1, (H, D))
        for h in range(H):
            at = (s // page)[:, None], h, (s % page // 16)[:, None]
            assert torch.equal(got_k[at[0], h, at[2], mk[s % 16]], want[:, h])
            assert torch.equal(got_v[at[0], h, at[2], mv[s % 16]], want[:, h])
