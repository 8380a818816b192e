"""pbd_paged_evict against a plain form: which slots stay, where the others go,
ties, protected slots, NaN and infinite weights, and what must not move."""
import math

import pytest
import torch

import paged_ref as ref
from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


class Call:
    def __init__(self, lens, keep, H, D, dtype, page=16, major="page", recent=0, sink=0, positions=True, weights="spread",
                 in_place=False, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.c = ref.Cache(lens, H, D, dtype, page=page, major=major, seed=seed)
        B, self.H, self.lens, self.keep, self.recent, self.sink = len(lens), H, lens, keep, recent, sink
        self.cap = self.c.width * page
        w = torch.exp(2 * torch.randn(B, H, self.cap, generator=g))
        if weights == "ties":
            w = torch.randint(0, 3, w.shape, generator=g).float()
        elif weights == "equal":
            w = torch.zeros_like(w)
        elif weights == "odd":      # NaN, infinities, both zeros, negative and subnormal values
            vals = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, -1.5, 1e-41, 2.0])
            w = vals[torch.randint(0, 8, w.shape, generator=g)]
        self.score0 = w
        self.pos0 = None
        if positions:
            self.pos0 = torch.stack([torch.stack([torch.randperm(2 * self.cap, generator=g)[: self.cap]
                                                  for _ in range(H)]) for _ in range(B)]).to(torch.int32)
        self.pos = [2 * n for n in lens]
        k, v, table = self.c.to(DEV)
        self.pool, self.before = (k, v), (k.clone().cpu(), v.clone().cpu())
        self.score = w.to(DEV)
        self.slot_pos = self.pos0.to(DEV) if positions else None
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.pages = pbd.make_pages(k, v, table, n_q_heads=H, head_dim=D, score=self.score, slot_pos=self.slot_pos,
                                    status=self.status)
        self.in_place = in_place
        self.score_out = None if in_place else torch.full_like(self.score, 77.0)
        self.pos_out = None if in_place or not positions else torch.full_like(self.slot_pos, 77)
        i = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
        self.dlens, self.dkeep, self.dpos = i(lens), i(keep), i(self.pos)
        self.new = self.dlens if in_place else i([-77] * B)
        n = pbd.pbd_paged_evict_workspace_bytes(self.pages, B, self.cap)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)

    def call(self):
        pbd.pbd_paged_evict(self.pages, self.dlens, self.cap, self.dkeep, self.new, self.ws, pos=self.dpos,
                            recent=self.recent, sink=self.sink, score_out=self.score_out, slot_pos_out=self.pos_out)

    def run(self):
        self.call()
        torch.cuda.synchronize()

    def check(self, skipped=()):
        k, v = (t.cpu() for t in self.pool)
        score = (self.score if self.in_place else self.score_out).cpu()
        pos = self.slot_pos if self.in_place else self.pos_out
        pos = None if pos is None else pos.cpu()
        bits = lambda t: t.contiguous().view(torch.int16 if t.dtype == BF else torch.int32)
        wk, wv = (t.clone() for t in self.before)
        ws = self.score0.clone() if self.in_place else torch.full_like(self.score0, 77.0)
        wp = None if pos is None else self.pos0.clone() if self.in_place else torch.full_like(self.pos0, 77)
        new = self.new.tolist()
        for b, n in enumerate(self.lens):
            if b in skipped:
                assert new[b] == (self.lens[b] if self.in_place else -77)
                continue
            keep = min(self.keep[b], n)
            assert new[b] == keep
            for h in range(self.H):
                p = None if self.pos0 is None else self.pos0[b, h].tolist()
                stay, moves = ref.kept(self.score0[b, h].tolist(), p, n, keep, self.pos[b] - self.recent, self.sink)
                ws[b, h, :keep] = self.score0[b, h, :keep]
                if wp is not None:
                    wp[b, h, :keep] = self.pos0[b, h, :keep]
                for to, fr in moves:
                    ws[b, h, to] = self.score0[b, h, fr]
                    if wp is not None:
                        wp[b, h, to] = self.pos0[b, h, fr]
                if moves:
                    to, fr = (torch.tensor(x) for x in zip(*moves))
                    (pt, ikt, ivt), (pf, ikf, ivf) = self.c.places(b, to), self.c.places(b, fr)
                    wk[pt[:, None], h, ikt] = self.before[0][pf[:, None], h, ikf]
                    wv[pt[:, None], h, ivt] = self.before[1][pf[:, None], h, ivf]
        assert torch.equal(bits(score), bits(ws))
        assert pos is None or torch.equal(pos, wp)
        assert torch.equal(bits(k), bits(wk)) and torch.equal(bits(v), bits(wv))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("weights", ["spread", "ties", "equal", "odd"])
def test_lengths_and_weights(weights, dtype, D):
    lens = [0, 1, 2, 15, 16, 17, 64, 100, 300, 300, 300]
    keep = [5, 1, 1, 8, 0, 16, 63, 10, 299, 300, 999]
    for in_place in (False, True):
        c = Call(lens, keep, 2, D, dtype, weights=weights, positions=weights != "ties", in_place=in_place, seed=D)
        c.run()
        c.check()
        assert int(c.status) == 0


@pytest.mark.parametrize("sink", [0, 30])
def test_positions_without_the_next_one(sink):
    """Positions kept, nothing recent protected: pos may be None, and then only the score and sink decide."""
    c = Call([200, 77, 2100], [100, 30, 500], 3, 64, BF, sink=sink, seed=sink + 3)
    c.dpos, c.pos = None, [math.inf] * 3
    c.run()
    c.check()
    assert int(c.status) == 0


@pytest.mark.parametrize("recent,sink", [(40, 0), (0, 30), (100, 20), (5000, 0), (0, 5000)])
def test_protected_slots(recent, sink):
    """Also more of them than stay."""
    c = Call([200, 77, 513], [100, 30, 500], 3, 64, BF, recent=recent, sink=sink, weights="odd", seed=recent)
    c.run()
    c.check()


@pytest.mark.parametrize("major", ["page", "head"])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_pages(page, major):
    c = Call([333, 1025, 16], [200, 600, 8], 2, 128, BF, page=page, major=major, recent=50, seed=page)
    c.run()
    c.check()


@pytest.mark.parametrize("n,keep", [(5000, 2500), (9001, 8990), (40003, 17), (70001, 35000)])
def test_long(n, keep):
    c = Call([n, n - 4321], [keep, keep], 2, 64, BF, page=64, recent=10, weights="spread" if n % 2 else "ties", seed=n)
    c.run()
    c.check()


def test_many_sequences():
    lens = [37 * i % 150 for i in range(70)]
    c = Call(lens, [i % 90 for i in range(70)], 4, 64, F32, seed=1)
    c.run()
    c.check()


def test_invalid_sequences_are_skipped():
    c = Call([100, 50, 60, 70], [30, 20, 20, 20], 2, 64, BF, recent=5)
    c.dlens = torch.tensor([100, -1, c.cap + 1, 70], dtype=torch.int32, device=DEV)
    c.dkeep = torch.tensor([30, 20, 20, -1], dtype=torch.int32, device=DEV)
    c.run()
    c.check(skipped=(1, 2, 3))
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY


def test_bad_pages_are_not_followed():
    c = Call([100, 100], [30, 30], 2, 64, BF)
    k, v, table = c.pages.keep[:3]
    t = table.clone()
    t[1, 6] = -1
    c.pages = pbd.make_pages(k, v, t, n_q_heads=2, head_dim=64, score=c.score, slot_pos=c.slot_pos, status=c.status)
    c.run()
    c.check(skipped=(1,))
    assert int(c.status) == pbd.PBD_STATUS_PAGE


def test_again_on_the_same_inputs_changes_nothing():
    c = Call([500, 300], [200, 299], 2, 64, BF, seed=4)
    for _ in range(3):
        c.run()
        c.check()


def test_captured_and_replayed():
    c = Call([500, 300], [200, 100], 2, 64, BF, recent=20, seed=6)
    c.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call()
    for keep in ([200, 100], [0, 500], [499, 1]):
        for t, t0 in zip(c.pool, c.before):
            t.copy_(t0.to(DEV))
        c.dkeep.copy_(torch.tensor(keep, dtype=torch.int32))
        c.keep = keep
        c.score_out.fill_(77.0)
        c.pos_out.fill_(77)
        g.replay()
        torch.cuda.synchronize()
        c.check()


def test_offsets_past_32_bits():
    """The last pages of pools of more than 2^31 elements move as a small pool's pages do."""
    c = Call([200, 90], [100, 41], 8, 128, BF, seed=4)
    first = [t.clone() for t in c.pool]
    c.run()
    c.check()
    n = 2 ** 31 // (8 * 128 * 16) + 40
    base = n - first[0].shape[0]
    far = [torch.empty(n, 8, 16 * 128, dtype=BF, device=DEV) for _ in range(2)]
    for f, s in zip(far, first):
        f[base:] = s
    table = c.pages.keep[2]
    c.pages = pbd.make_pages(*far, torch.where(table < 0, table, table + base), n_q_heads=8, head_dim=128,
                             score=c.score, slot_pos=c.slot_pos, status=c.status)
    c.run()
    assert int(c.status) == 0
    for f, s in zip(far, c.pool):
        assert torch.equal(f[base:].view(torch.int16), s.view(torch.int16))
