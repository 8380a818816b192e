"""pbd_paged_append against a plain form in 64 bits: rows per call, where a block
begins, types, norms, strides, slot state, and what must stay as it was."""
import math

import pytest
import torch

import paged_ref as ref
from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"
U = ref.U


def rope_table(n, D, theta=1e6):
    ang = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    return torch.stack((ang.cos(), ang.sin()), -1).float()


def rotated(x, gain, rope, eps):
    """64-bit norm and rotation of [rows][heads][D]; and the fp32 result's bound: the mean square's D terms,
    the root and quotient, two products of the norm, two of the rotation and their sum, of |a| + |b|."""
    D = x.shape[-1]
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    a, b = x[..., : D // 2], x[..., D // 2:]
    c, s = rope[:, None, :, 0].double(), rope[:, None, :, 1].double()
    tol = ((D if gain is not None else 0) + 12) * U * torch.cat((a.abs() + b.abs(),) * 2, -1)
    return torch.cat((a * c - b * s, b * c + a * s), -1), tol


def half_step(x, dtype):
    return x.abs() * (torch.finfo(dtype).eps / 2) + 1e-30


class Call:
    def __init__(self, lens, n_new, rows, H, G, D, dtype, page=16, major="page", norm=True, with_q=True, state=True,
                 joined=True, seed=0, pos=None):
        g = torch.Generator().manual_seed(seed)
        B, HQ = len(lens), H * G
        self.c = ref.Cache(lens, H, D, dtype, page=page, major=major, seed=seed, room=rows)
        self.B, self.R, self.H, self.HQ, self.D, self.dtype = B, rows, H, HQ, D, dtype
        self.lens, self.n_new = lens, n_new
        x = torch.randn(B, rows, (HQ + 2 * H) * D, generator=g) * 3
        for b in range(B):
            if n_new is not None:
                x[b, max(0, n_new[b]):] = math.nan                           # rows past n_new are not read
        self.q, self.k, self.v = x[..., : HQ * D], x[..., HQ * D: (HQ + H) * D], x[..., (HQ + H) * D:]
        dx = x.to(DEV)
        cut = (dx[..., : HQ * D], dx[..., HQ * D: (HQ + H) * D], dx[..., (HQ + H) * D:])
        if not joined:
            assert HQ == H
            cut = tuple(t.contiguous() for t in cut)
        self.dq, self.dk, self.dv = cut
        if not with_q:
            self.dq = None
        self.gains = [(1 + 0.1 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in range(2)]
        self.pos = pos if pos is not None else [n + 5 for n in lens]
        self.rope = rope_table(max(max(self.pos), 0) + rows, D)
        k, v, table = self.c.to(DEV)
        self.k0, self.v0 = k.clone(), v.clone()
        cap = self.c.width * page
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.score = torch.full((B, H, cap), 3.0, device=DEV) if state else None
        self.slot_pos = torch.full((B, H, cap), -9, dtype=torch.int32, device=DEV) if state else None
        self.pool = (k, v)
        self.pages = pbd.make_pages(k, v, table, n_q_heads=HQ, head_dim=D, score=self.score, slot_pos=self.slot_pos,
                                    status=self.status)
        self.q_out = torch.full((B, rows, HQ * D), 77.0, device=DEV) if with_q else None
        self.len_out = torch.full((B,), -77, dtype=torch.int32, device=DEV)
        self.i = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device=DEV)

    def run(self):
        dev = [None if t is None else t.to(DEV) for t in self.gains]
        self.keep = dev
        pbd.pbd_paged_append(self.pages, self.dk, self.dv, self.i(self.lens), self.i(self.pos), self.rope.to(DEV),
                             q=self.dq, q_out=self.q_out, n_new=self.i(self.n_new),
                             q_norm=dev[0] if self.dq is not None else None, k_norm=dev[1], eps=1e-6,
                             len_out=self.len_out)
        torch.cuda.synchronize()

    def check(self, skipped=()):
        k, v = (t.cpu() for t in self.pool)
        # the pool as it has to be, with NaN where a new value belongs; everything else bit for bit
        wk, wv = self.k0.cpu().clone(), self.v0.cpu().clone()
        for b in range(self.B):
            n = self.R if self.n_new is None else self.n_new[b]
            if b in skipped:
                assert int(self.len_out[b]) == -77
                if self.q_out is not None:
                    assert torch.all(self.q_out[b] == 77.0)
                if self.score is not None:
                    assert torch.all(self.score[b] == 3.0) and torch.all(self.slot_pos[b] == -9)
                continue
            first = self.lens[b]
            assert int(self.len_out[b]) == first + n
            at = self.rope[self.pos[b]: self.pos[b] + n]
            want, tol = rotated(self.k[b, :n].unflatten(1, (self.H, self.D)), self.gains[1], at, 1e-6)
            page, ik, iv = self.c.places(b, torch.arange(first, first + n))
            value = self.v[b, :n].unflatten(1, (self.H, self.D))
            for h in range(self.H):
                got = k[page[:, None], h, ik].double()
                assert torch.all((got - want[:, h]).abs() <= tol[:, h] + half_step(want[:, h], self.dtype) * 1.01)
                assert torch.equal(v[page[:, None], h, iv], value[:, h].to(self.dtype))
                wk[page[:, None], h, ik] = k[page[:, None], h, ik]
                wv[page[:, None], h, iv] = v[page[:, None], h, iv]
            if self.q_out is not None:
                wq, tq = rotated(self.q[b, :n].unflatten(1, (self.HQ, self.D)), self.gains[0], at, 1e-6)
                got = self.q_out[b].double().cpu().unflatten(1, (self.HQ, self.D))
                assert torch.all((got[:n] - wq).abs() <= tq + half_step(wq, F32))
                assert torch.all(got[n:] == 77.0)
            if self.score is not None:
                s, p = self.score[b].cpu(), self.slot_pos[b].cpu()
                assert torch.all(s[:, first: first + n] == 0)
                want_pos = torch.arange(self.pos[b], self.pos[b] + n, dtype=torch.int32)
                assert torch.all(p[:, first: first + n] == want_pos)
                s[:, first: first + n], p[:, first: first + n] = 3.0, -9
                assert torch.all(s == 3.0) and torch.all(p == -9)
        bits = torch.int16 if self.dtype == BF else torch.int32
        assert torch.equal(k.contiguous().view(bits), wk.contiguous().view(bits))
        assert torch.equal(v.contiguous().view(bits), wv.contiguous().view(bits))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 2, 7, 8, 16, 33, 100, 333])
def test_rows(rows, dtype, D):
    """Few rows and many, from every place of a block, each sequence with its own count (none, too)."""
    lens = [0, 1, 3, 15, 16, 30]
    c = Call(lens, [rows, 0, max(0, rows - 1), rows, (rows + 1) // 2, rows], rows, 2, 2, D, dtype, seed=rows)
    c.run()
    c.check()
    assert int(c.status) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [1, 7, 9])
def test_many_sequences(rows, D):
    """Few rows of many sequences, inside one block and over its end."""
    lens = [(7 * i) % 50 for i in range(560)]
    c = Call(lens, [(rows, rows - 1, rows)[i % 3] for i in range(560)], rows, 2, 2, D, BF, seed=rows)
    c.run()
    c.check()
    assert int(c.status) == 0


@pytest.mark.parametrize("rows", [4, 300])
def test_no_rows(rows):
    c = Call([3, 17], [0, 0], rows, 2, 2, 64, BF)
    c.run()
    c.check()


@pytest.mark.parametrize("H,G", [(1, 1), (3, 5), (8, 2), (1, 33)])
@pytest.mark.parametrize("rows", [1, 20, 300])
def test_heads(H, G, rows):
    c = Call([4, 13], None, rows, H, G, 128, BF, seed=G)
    c.run()
    c.check()


@pytest.mark.parametrize("major", ["page", "head"])
@pytest.mark.parametrize("page", [16, 64, 512])
def test_pages(page, major):
    for rows in (3, 70, 210):
        c = Call([5, 700, 48], [rows, rows, 1], rows, 2, 1, 64, BF, page=page, major=major)
        c.run()
        c.check()


@pytest.mark.parametrize("rows", [1, 9, 290])
def test_without_norm_queries_or_state(rows):
    for kw in (dict(norm=False), dict(with_q=False), dict(state=False), dict(joined=False)):
        c = Call([4, 40], None, rows, 2, 1, 64, F32, **kw)
        c.run()
        c.check()


def test_far_positions():
    c = Call([4], None, 2, 1, 1, 128, BF, pos=[131000])
    c.run()
    c.check()


@pytest.mark.parametrize("rows", [2, 20, 120])
def test_sequences_that_do_not_fit_are_skipped(rows):
    """No room in the table, a negative length or count, positions outside the rope table."""
    c = Call([0, 10, 4, 20, 8], None, rows, 2, 2, 64, BF)
    full = c.c.width * c.c.page
    c.lens = [0, full - rows + 1, -1, 20, 8]
    c.n_new = [rows, rows, rows, rows + 1, rows]
    c.pos = [0, 0, 0, 0, c.rope.shape[0] - rows + 1]
    c.run()
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY
    c.n_new = [rows] * 5
    c.check(skipped=(1, 2, 3, 4))


@pytest.mark.parametrize("rows", [2, 40, 290])
def test_bad_pages_are_not_followed(rows):
    c = Call([3, 14], None, rows, 2, 1, 64, BF)
    k, v, table = c.pages.keep[:3]
    t = table.clone()
    t[1, (14 + rows - 1) // 16] = c.pages.n_pages
    c.pages = pbd.make_pages(k, v, t, n_q_heads=2, head_dim=64, score=c.score, slot_pos=c.slot_pos, status=c.status)
    c.run()
    assert int(c.status) == pbd.PBD_STATUS_PAGE
    c.check(skipped=(1,))


def test_slots_past_the_state_do_not_fit():
    """score and slot_pos shorter than the table bound the cache."""
    c = Call([10], None, 8, 1, 1, 64, BF)
    k, v, table = c.pages.keep[:3]
    c.score, c.slot_pos = c.score[:, :, :17].contiguous(), c.slot_pos[:, :, :17].contiguous()
    c.pages = pbd.make_pages(k, v, table, n_q_heads=1, head_dim=64, score=c.score, slot_pos=c.slot_pos, status=c.status)
    c.run()
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY
    c.check(skipped=(0,))


@pytest.mark.parametrize("rows", [2, 300])
def test_captured_and_replayed(rows):
    """A replay appends what the buffers hold by then, at the lengths of then."""
    c = Call([8, 35], None, rows, 2, 2, 64, BF)                  # (its table has pages for these)
    first = c.i(c.lens)
    pos, rope, gains = c.i(c.pos), rope_table(1000, 64).to(DEV), [g.to(DEV) for g in c.gains]
    c.rope = rope.cpu()

    def call():
        pbd.pbd_paged_append(c.pages, c.dk, c.dv, first, pos, rope, q=c.dq, q_out=c.q_out, q_norm=gains[0],
                             k_norm=gains[1], eps=1e-6, len_out=c.len_out)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for c.lens in ([3, 30], [8, 35], [3, 30]):
        first.copy_(c.i(c.lens))
        c.pool[0].copy_(c.k0)
        c.pool[1].copy_(c.v0)
        c.score.fill_(3.0)
        c.slot_pos.fill_(-9)
        g.replay()
        torch.cuda.synchronize()
        c.check()


def test_two_streams():
    """Calls on two streams, each on its own cache and tensors."""
    calls = [Call([4, 13], None, rows, 2, 2, 64, BF, seed=rows) for rows in (5, 290)]
    streams = [torch.cuda.Stream() for _ in calls]
    args = [(c.i(c.lens), c.i(c.pos), c.rope.to(DEV), [g.to(DEV) for g in c.gains]) for c in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s, (lens, pos, rope, gains) in zip(calls, streams, args):
            with torch.cuda.stream(s):
                pbd.pbd_paged_append(c.pages, c.dk, c.dv, lens, pos, rope, q=c.dq, q_out=c.q_out, q_norm=gains[0],
                                     k_norm=gains[1], eps=1e-6, len_out=c.len_out)
    torch.cuda.synchronize()
    for c in calls:
        c.check()


@pytest.mark.parametrize("rows", [2, 300])
def test_offsets_past_32_bits(rows):
    """The last pages of pools of more than 2^31 elements take what a small pool's pages take."""
    c = Call([3, 30], None, rows, 8, 1, 128, BF)
    c.run()
    small, n = c.pool, 2 ** 31 // (8 * 128 * 16) + 40
    base = n - small[0].shape[0]
    far = [torch.empty(n, 8, 16 * 128, dtype=BF, device=DEV) for _ in range(2)]
    for f, first in zip(far, (c.k0, c.v0)):
        f[base:] = first
    table = c.pages.keep[2]
    c.pages = pbd.make_pages(*far, torch.where(table < 0, table, table + base), n_q_heads=8, head_dim=128,
                             status=c.status)
    c.run()
    assert int(c.status) == 0
    for f, s in zip(far, small):
        assert torch.equal(f[base:].view(torch.int16), s.view(torch.int16))
