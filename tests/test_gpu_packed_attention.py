"""pbd_packed_attention and pbd_tree_attention against a plain form in 64 bits: rows and lengths from none to long ones,
head layouts, pages, strides, both types, masks that leave rows empty, and what must not be read."""
import math

import pytest
import torch

import paged_ref as ref
import rows_ref as rr
from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


class Call:
    """One cache, packed rows of its sequences and outputs on the GPU.  trees: parents of each sequence's rows, masks: their
    masks; neither: causal rows."""

    def __init__(self, cache, counts, G, trees=None, masks=None, max_len=None, q_pad=0, more=3, seed=1, gain=1.0):
        g = torch.Generator().manual_seed(seed)
        self.cache, self.counts, self.B, HQ = cache, counts, len(counts), cache.H * G
        self.starts = rr.starts(counts)
        self.R = max(1, self.starts[-1] + more)
        self.HQ, self.D = HQ, cache.D
        self.q = (torch.randn(self.R, HQ, cache.D, generator=g) * gain).to(cache.dtype)
        k, v, table = cache.to(DEV)
        self.max_len = max_len or cache.width * cache.page
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.pages = pbd.make_pages(k, v, table, n_q_heads=HQ, head_dim=cache.D, status=self.status)
        flat = torch.full((self.R, HQ * cache.D + q_pad), math.nan, dtype=cache.dtype, device=DEV)
        flat[:, : HQ * cache.D] = self.q.to(DEV).flatten(1)
        self.dq = flat[:, : HQ * cache.D].unflatten(1, (HQ, cache.D))
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
        self.lens, self.row_start = i32(cache.lens), i32(self.starts)
        self.out = torch.full((self.R, HQ, cache.D), 77.0, dtype=cache.dtype, device=DEV)
        self.lse = torch.full((self.R, HQ), 77.0, device=DEV)
        if trees is not None:
            masks = [rr.ancestors(t) for t in trees]
        self.masks = masks
        self.mask = None
        if masks is not None:
            flat = [m for row in masks for m in row] + [-1 & (1 << 64) - 1] * (self.R - self.starts[-1])
            self.mask = rr.to_i64(flat).to(DEV)
        size = pbd.pbd_packed_attention_workspace_bytes if masks is None else pbd.pbd_tree_attention_workspace_bytes
        n = size(self.pages, self.B, self.R, self.max_len)
        assert n > 0
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)      # NaN wherever it is read unwritten

    def enqueue(self, **kw):
        if self.mask is None:
            pbd.pbd_packed_attention(self.pages, self.dq, self.row_start, self.lens, self.max_len, self.out, self.ws,
                                     lse=self.lse, **kw)
        else:
            pbd.pbd_tree_attention(self.pages, self.dq, self.row_start, self.lens, self.mask, self.max_len, self.out,
                                   self.ws, lse=self.lse, **kw)

    def run(self, **kw):
        self.enqueue(**kw)
        torch.cuda.synchronize()

    def see(self, b):
        n, length = self.counts[b], self.cache.lens[b]
        return rr.causal(n, length) if self.masks is None else rr.by_mask(self.masks[b], length)

    def check(self, scale=None, skip=()):
        out, lse = self.out.double().cpu(), self.lse.double().cpu()
        for b, n in enumerate(self.counts):
            rows = slice(self.starts[b], self.starts[b] + n)
            if b in skip:
                assert torch.all(out[rows] == 77.0) and torch.all(lse[rows] == 77.0)
                continue
            if n == 0:
                continue
            o, s, o_tol, s_tol = rr.attention(self.cache, b, self.q[rows], self.see(b), scale or self.D ** -0.5)
            off = (out[rows] - o).abs()
            assert torch.all(off <= o_tol), (b, n, self.cache.lens[b], off.max(), (off - o_tol).argmax())
            none = s == -math.inf
            assert torch.equal(lse[rows] == -math.inf, none)
            assert torch.all(out[rows][none] == 0)
            assert torch.all((lse[rows] - s)[~none].abs() <= s_tol[~none]), (b, n)
        assert torch.all(out[self.starts[-1]:] == 77.0) and torch.all(lse[self.starts[-1]:] == 77.0)


# (slots, rows of them): whole prompts, chunks, one row, none
SIZES = [(0, 0), (1, 1), (5, 5), (15, 15), (16, 16), (17, 17), (31, 31), (33, 33), (64, 64), (65, 65), (100, 1), (129, 64),
         (200, 33), (77, 0), (300, 300), (513, 129)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_sizes(dtype, D):
    for pick in (SIZES, SIZES[:8], SIZES[-2:]):          # (many, few and long rows a sequence: each tile count)
        c = Call(ref.Cache([m for m, _ in pick], 2, D, dtype, seed=D), [n for _, n in pick], 2)
        c.run()
        c.check()
        assert int(c.status) == 0


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (8, 2), (2, 5), (2, 8), (1, 16), (1, 17), (1, 40), (1, 80)])
def test_head_layouts(H, G):
    for dtype, D in ((BF, 128), (F32, 64)):
        c = Call(ref.Cache([200, 77, 33], H, D, dtype, seed=G), [50, 77, 1], G)
        c.run()
        c.check()


@pytest.mark.parametrize("page", [16, 32, 64, 256, 4096])
@pytest.mark.parametrize("major", ["page", "head"])
def test_pages_and_strides(page, major):
    c = Call(ref.Cache([130, 1, 0, 259], 3, 64, BF, page=page, major=major, seed=page), [70, 1, 0, 259], 4, q_pad=16)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,H,D", [(BF, 2, 128), (F32, 1, 64)])
@pytest.mark.parametrize("sizes", [[(4096, 1)], [(5000, 40)], [(3001, 700)], [(9000, 17), (8000, 3), (20, 20)], [(2049, 2049)]])
def test_long(dtype, H, D, sizes):
    """Few rows over many slots (split) and many rows, lengths ragged."""
    c = Call(ref.Cache([m for m, _ in sizes], H, D, dtype, page=64, seed=len(sizes)), [n for _, n in sizes], 2)
    c.run()
    c.check()


def test_many_sequences():
    """More sequences than a wave looks at in one step."""
    sizes = [(1 + b % 40, b % 5 if b % 40 + 1 >= b % 5 else 1) for b in range(300)]
    c = Call(ref.Cache([m for m, _ in sizes], 1, 64, BF, seed=2), [n for _, n in sizes], 2)
    c.run()
    c.check()


def test_a_bound_longer_than_any_sequence():
    c = Call(ref.Cache([5, 40], 2, 128, BF, room=5000), [5, 7], 2, more=500)
    assert c.max_len > 5000
    c.run()
    c.check()


@pytest.mark.parametrize("trees", [False, True])
def test_sharp_and_flat_weights(trees):
    """Scores up to some hundreds (one slot takes all) and of 0 (equal weights)."""
    g = torch.Generator().manual_seed(4)
    for gain in (0.0, 40.0):
        for dtype in (BF, F32):
            t = [rr.random_tree(n, g) for n in (1, 30, 64)] if trees else None
            c = Call(ref.Cache([1, 100, 1000], 2, 128, dtype, seed=5), [1, 30, 64], 4, trees=t, gain=gain)
            c.run()
            c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,G", [(2, 2), (1, 8), (2, 1)])
def test_trees(dtype, D, H, G):
    g = torch.Generator().manual_seed(D)
    sizes = [(1, 1), (64, 64), (63, 63), (65, 64), (17, 17), (400, 17), (1000, 33), (50, 0), (700, 64)]
    c = Call(ref.Cache([m for m, _ in sizes], H, D, dtype, seed=D), [n for _, n in sizes], G,
             trees=[rr.random_tree(n, g) for _, n in sizes])
    c.run()
    c.check()
    assert int(c.status) == 0


def test_masks_of_any_kind():
    """No bits at all with and without slots before the tree, all bits, bits past the tree, later nodes."""
    full = (1 << 64) - 1
    masks = [[0, full, 1, 0b100], [0, 0, full], [full] * 33, [1 << 63, 0, full ^ 1], [1 << (63 - i) for i in range(64)]]
    lens = [4, 40, 33, 1030, 64]
    for dtype, D in ((BF, 128), (BF, 64), (F32, 128)):
        c = Call(ref.Cache(lens, 2, D, dtype, seed=3), [len(m) for m in masks], 3, masks=masks)
        c.run()
        c.check()


@pytest.mark.parametrize("B,n,t", [(1, 4096, 17), (1, 33001, 5), (3, 9000, 64), (40, 700, 20)])
def test_trees_over_long_caches(B, n, t):
    g = torch.Generator().manual_seed(n)
    lens = [n - 17 * b for b in range(B)]
    c = Call(ref.Cache(lens, 2, 128, BF, page=64, seed=n), [t] * B, 2, trees=[rr.random_tree(t, g) for _ in lens])
    c.run()
    c.check()


def test_a_causal_mask_is_the_causal_rows():
    sizes = [(64, 64), (500, 33)]
    lens, counts = [m for m, _ in sizes], [n for _, n in sizes]
    cache = ref.Cache(lens, 2, 128, BF, seed=8)
    a = Call(cache, counts, 2)
    b = Call(cache, counts, 2, masks=[[(1 << i + 1) - 1 for i in range(n)] for n in counts])
    a.run()
    b.run()
    a.check()
    b.check()


@pytest.mark.parametrize("rows", [64, 20, 9])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128)])
@pytest.mark.parametrize("trees", [False, True])
def test_hidden_values_that_are_not_finite(trees, dtype, D, rows):
    """Infinite and NaN keys and values of slots that some rows of a tile do not see: those rows are as if they were
    finite, the others get what fp32 arithmetic makes of them."""
    length = 100 + rows
    cache = ref.Cache([length, length], 2, D, dtype, seed=rows)
    first = length - rows
    clean_k, clean_v = cache.dk.clone(), cache.dv.clone()
    at = first + rows // 2
    for b in range(2):
        cache.dv[b, 0, at, 3] = math.nan
        cache.dv[b, 0, at, 7] = math.inf
        cache.dv[b, 1, at, D - 1] = -math.inf
        cache.dv[b, 1, length - 1, 0] = math.inf
        if b == 1:
            cache.dk[b, 1, length - 1, 5] = math.nan
        cache.put(b, 0, cache.dk[b, :, :length], cache.dv[b, :, :length])
    masks = None
    if trees:
        line = [(1 << i + 1) - 1 for i in range(rows)]
        masks = [line, line]
    c = Call(cache, [rows, rows], 2, masks=masks)
    c.run()
    out = c.out.double().cpu().view(2, rows, 2, 2, D) if c.out.shape[0] == 2 * rows else \
        c.out.double().cpu()[: 2 * rows].view(2, rows, 2, 2, D)
    dirty_k, dirty_v = cache.dk, cache.dv
    cache.dk, cache.dv = clean_k, clean_v
    half, last = rows // 2, rows - 1
    for b in range(2):
        q = c.q[b * rows: (b + 1) * rows]
        o, _, tol, _ = rr.attention(cache, b, q, c.see(b), D ** -0.5)
        o, tol = o.view(rows, 2, 2, D), tol.view(rows, 2, 2, D)
        ok = torch.ones(rows, 2, 2, D, dtype=torch.bool)
        ok[half:, 0, :, 3] = ok[half:, 0, :, 7] = False
        ok[half:, 1, :, D - 1] = False
        ok[last, 1, :, 0] = False
        if b == 1:
            ok[last, 1] = False
        assert torch.all(((out[b] - o).abs() <= tol)[ok])
        assert torch.isnan(out[b][half:, 0, :, 3]).all()
        assert torch.all(out[b][half:, 0, :, 7] == math.inf)
        end = last if b == 1 else rows
        assert torch.all(out[b][half: end, 1, :, D - 1] == -math.inf)
        if b == 0:
            assert torch.all(out[b][last, 1, :, 0] == math.inf)
        else:
            assert torch.isnan(out[b][last, 1]).all()
    cache.dk, cache.dv = dirty_k, dirty_v


def test_infinite_keys():
    """A score of -inf has weight 0; one of +inf makes its rows NaN, and theirs alone."""
    for dtype in (BF, F32):
        cache = ref.Cache([50], 1, 64, dtype, seed=1)
        cache.dk[0, 0, 10, 4] = math.inf
        cache.put(0, 0, cache.dk[0, :, :50], cache.dv[0, :, :50])
        c = Call(cache, [50], 1)
        c.run()
        out = c.out.double().cpu()[:50, 0]
        up = (c.q[:50, 0, 4].double() > 0) & (torch.arange(50) >= 10)
        assert torch.isnan(out[up]).all() and torch.isfinite(out[~up]).all()
        see = rr.causal(50, 50)
        see[:, 10] = False
        cache.dk[0, 0, 10, 4] = 0.0
        o, _, tol, _ = rr.attention(cache, 0, c.q[:50], see, 64 ** -0.5)
        assert torch.all(((out - o[:, 0]).abs() <= tol[:, 0])[~up])


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128)])
@pytest.mark.parametrize("step", [1.0, -1.0, 0.25, 3.0])
def test_rising_and_falling_scores(dtype, D, step):
    """Scores that grow or fall all along the slots: slowly, so that weights grow to many times the first ones' before the
    reference follows, and fast."""
    cache = ref.Cache([200, 180, 1500], 1, D, dtype, seed=2)
    for b, m in enumerate(cache.lens):
        cache.dk[b, 0, :m] = 0.0
        cache.dk[b, 0, :m, 0] = (torch.arange(m) % 200).to(dtype)
        cache.put(b, 0, cache.dk[b, :, :m], cache.dv[b, :, :m])
    c = Call(cache, [200, 30, 3], 2)
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = step
    c.dq.copy_(c.q.to(DEV))
    for scale in (0.2, 0.7):
        c.out.fill_(77.0)
        c.lse.fill_(77.0)
        c.run(scale=scale)
        c.check(scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("odd", [False, True])
def test_scores_of_any_size(dtype, odd):
    """Scores of 1e30 in either sign, the largest ones last, first, or followed by scores of 0: the highest slots share all,
    also where the last slot's NaN, hidden from the rows before, sends the tile through a second pass.

    Weights of 1 and 0 are exact in either type: n roundings of the sum and two of the quotient, below U sum |v| / count each,
    and the output's own."""
    D, n = 64, 150
    cache = ref.Cache([n] * 6, 1, D, dtype, seed=6)
    ramp = torch.arange(n) % 128
    for b, k in enumerate((1.0 + ramp, 1.0 - ramp, -400.0 + ramp, 400.0 - ramp, -1.0 * (ramp < 40), 1.0 * (ramp < 40))):
        cache.dk[b, 0, :n] = 0.0
        cache.dk[b, 0, :n, 0] = k.to(dtype)
        if odd:
            cache.dv[b, 0, n - 1] = math.nan
        cache.put(b, 0, cache.dk[b, :, :n], cache.dv[b, :, :n])
    c = Call(cache, [n] * 6, 1)
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 2.0 ** 92
    c.dq.copy_(c.q.to(DEV))
    c.run()
    out = c.out.double().cpu()
    for b in range(6):
        k, v = cache.dk[b, 0, :n, 0].double(), cache.dv[b, 0].double()
        for i in range(n):
            if odd and i == n - 1:
                assert torch.isnan(out[b * n + i, 0]).all()
                continue
            top = (k[: i + 1] == k[: i + 1].max()).nonzero()[:, 0]
            want = v[top].mean(0)
            tol = want.abs() * torch.finfo(dtype).eps / 2 * 1.01 + (n + 2) * ref.U * v[top].abs().mean(0)
            assert torch.all((out[b * n + i, 0] - want).abs() <= tol), (b, i)


def test_queries_that_are_not_finite_stay_in_their_rows():
    """The others keep the bound.  (Those of the same 32 may differ in their last bits: their weights are rounded against the
    whole row's maximum where the tile is gone over again, and against an earlier one where not.)"""
    for dtype in (BF, F32):
        c = Call(ref.Cache([200, 40], 2, 64, dtype, seed=7), [60, 40], 2)
        q = c.q.clone()
        bad = [(3, 1), (59, 0), (70, 3)]
        for r, h in bad:
            q[r, h, 5] = math.nan
        c.dq.copy_(q.to(DEV))
        c.run()
        out, lse = c.out.clone(), c.lse.clone()
        c.dq.copy_(c.q.to(DEV))
        c.run()
        for r, h in bad:
            assert torch.isnan(out[r, h]).all() and torch.isnan(lse[r, h])
            out[r, h], lse[r, h] = c.out[r, h], c.lse[r, h]
        c.check()
        c.out.copy_(out)
        c.lse.copy_(lse)
        c.check()


def test_two_streams_at_once():
    g = torch.Generator().manual_seed(3)
    a = Call(ref.Cache([3000, 40], 2, 128, BF, seed=1), [33, 40], 2)
    b = Call(ref.Cache([900, 64], 2, 128, BF, seed=2), [17, 64], 2, trees=[rr.random_tree(17, g), rr.random_tree(64, g)])
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        a.enqueue(stream=side[0])
        b.enqueue(stream=side[1])
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_scale_and_stream():
    c = Call(ref.Cache([100, 40], 2, 128, BF), [30, 40], 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(scale=0.3, stream=side)
    side.synchronize()
    c.check(scale=0.3)


def test_without_lse():
    c = Call(ref.Cache([100, 2000], 2, 128, BF), [30, 2], 2)
    c.run()
    want = c.out.clone()
    c.out.fill_(77.0)
    pbd.pbd_packed_attention(c.pages, c.dq, c.row_start, c.lens, c.max_len, c.out, c.ws)
    assert torch.equal(want, c.out)


def test_bitwise_the_same_again_and_beside_other_sequences():
    cache = ref.Cache([500, 77, 1200], 2, 128, BF, seed=3)
    c = Call(cache, [40, 30, 50], 2)
    c.run()
    first = c.out.clone()
    c.ws.fill_(0xFF)
    c.run()
    assert torch.equal(first, c.out)
    c.lens = torch.tensor([100, 77, 60], dtype=torch.int32, device=DEV)
    c.run()
    assert torch.equal(first[40:70], c.out[40:70])


def test_shared_pages():
    """Sequences over the same prefix pages, of different lengths."""
    cache = ref.Cache([300, 300], 2, 128, BF, seed=9)
    cache.table[1] = cache.table[0]
    cache.dk[1], cache.dv[1] = cache.dk[0], cache.dv[0]
    cache.lens = [300, 123]
    c = Call(cache, [20, 100], 2)
    c.run()
    c.check()


@pytest.mark.parametrize("trees", [False, True])
def test_offsets_past_32_bits(trees):
    """A pool of more than 2^31 elements (2^32 bytes), its last pages in use."""
    H, D, page, n = 8, 128, 64, 2 ** 31 // (8 * 128 * 64) + 40
    small = ref.Cache([1000], H, D, BF, page=page, seed=11)
    k = torch.empty(n, H, page * D, dtype=BF, device=DEV)
    v = torch.empty(n, H, page * D, dtype=BF, device=DEV)
    last = torch.arange(n - small.width, n)
    for pool, src in ((k, small.k), (v, small.v)):
        pool[last] = src[small.table[0].long()].to(DEV)
    g = torch.Generator().manual_seed(1)
    c = Call(small, [60], 2, trees=[rr.random_tree(60, g)] if trees else None)
    c.pages = pbd.make_pages(k, v, last.to(torch.int32).to(DEV).view(1, -1), n_q_heads=2 * H, head_dim=D, status=c.status)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype,H,G,D", [(BF, 8, 2, 64), (BF, 4, 8, 128), (BF, 12, 3, 64), (F32, 12, 5, 64)])
@pytest.mark.parametrize("B", [2, 17, 64])
def test_many_groups_of_ragged_sequences(dtype, H, G, D, B):
    """513 to 4096 work-groups over sequences of 1024 slots and more, which are taken by length: every row comes once,
    whatever the others are, none at all or out of range among them."""
    g = torch.Generator().manual_seed(B + H)
    draw = lambda hi: int(torch.randint(0, hi + 1, (1,), generator=g))
    R = 90000 // (G * H)
    counts = [draw(2 * R // B) if b % 7 != 3 else 0 for b in range(B)] if B > 2 else [R // 2, R // 2 - 50]
    lens = [n + (700 + draw(900) if b % 3 else 0) for b, n in enumerate(counts)]
    c = Call(ref.Cache(lens, H, D, dtype, page=64, seed=B), counts, G)
    assert (c.R * G // 128 + B) * H > 512 and (c.R * G // 64 + B) * H <= 4096
    assert c.max_len - c.R / B / 2 >= 1024
    c.run()
    c.check()
    assert int(c.status) == 0
    bad = [b for b, n in enumerate(counts) if n and b % 5 == 1]
    c.lens = torch.tensor([[-1, n - 1, 10 ** 6][b % 3] if b in bad else m for b, (m, n) in enumerate(zip(lens, counts))],
                          dtype=torch.int32, device=DEV)
    want = c.out.clone(), c.lse.clone()
    c.out.fill_(77.0)
    c.lse.fill_(77.0)
    c.run()
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY
    for b, n in enumerate(counts):
        rows = slice(c.starts[b], c.starts[b] + n)
        for got, was in zip((c.out, c.lse), want):
            assert torch.all(got[rows] == 77.0) if b in bad else torch.equal(got[rows], was[rows])


@pytest.mark.parametrize("long", [False, True])
def test_lengths_and_rows_out_of_range_skip_the_sequence(long):
    m = 3000 if long else 100
    for lens, bad in (([m, m + 10 ** 6, 50, 60], (1,)), ([m, -1, 50, 60], (1,)), ([m, 60, 4, 60], (2,))):
        c = Call(ref.Cache([m, 60, 50, 60], 2, 64, BF), [9, 10, 5, 60], 2)
        c.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        c.run()
        c.check(skip=bad)
        assert int(c.status) == pbd.PBD_STATUS_CAPACITY


def test_rows_past_the_bound_skip_the_sequence():
    c = Call(ref.Cache([30, 20], 2, 64, BF), [10, 8], 2, more=0)
    for bad in ([0, 10, 19], [-3, 10, 18], [0, 10, 2 ** 31 - 1], [0, 10, 9]):
        c.out.fill_(77.0)
        c.lse.fill_(77.0)
        c.status.zero_()
        c.row_start = torch.tensor(bad, dtype=torch.int32, device=DEV)
        c.run()
        assert int(c.status) == pbd.PBD_STATUS_CAPACITY, bad
        if bad[0] == 0:
            c.check(skip=(1,))
        else:
            assert torch.all(c.out[:10] == 77.0)


def test_trees_of_more_than_64_nodes_are_skipped():
    c = Call(ref.Cache([100, 30], 2, 64, BF), [65, 10], 2, masks=[[1] * 65, [3] * 10])
    c.run()
    c.check(skip=(0,))
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY


@pytest.mark.parametrize("rows", [60, 5])
def test_bad_pages_skip_the_sequence(rows):
    """Wherever the page lies: also where a tile of rows, or a split of the slots, does not reach."""
    c = Call(ref.Cache([100, 1100], 2, 64, BF), [20, rows], 2)
    k, v, table = c.pages.keep[:3]
    for where in (0, 40, 68):
        for bad in (-1, k.shape[0], 2 ** 31 - 1, -2 ** 31):
            t = table.clone()
            t[1, where] = bad
            c.status.zero_()
            c.out.fill_(77.0)
            c.lse.fill_(77.0)
            c.pages = pbd.make_pages(k, v, t, n_q_heads=4, head_dim=64, status=c.status)
            c.run()
            c.check(skip=(1,))
            assert int(c.status) == pbd.PBD_STATUS_PAGE


def test_two_graphs_replayed_in_turn():
    """Captured calls with workspaces of their own, replayed between eager work, inputs changed in place."""
    g = torch.Generator().manual_seed(6)
    a = Call(ref.Cache([700, 40], 2, 128, BF, seed=1), [33, 40], 2)
    b = Call(ref.Cache([900, 64], 2, 128, BF, seed=2), [17, 64], 2, trees=[rr.random_tree(17, g), rr.random_tree(64, g)])
    graphs = []
    for c in (a, b):
        c.run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.enqueue()
        graphs.append(graph)
    for turn in range(3):
        for c, graph in zip((a, b), graphs):
            new = torch.randn(c.R, c.HQ, c.D, generator=g).to(BF)
            c.q = new
            c.dq.copy_(new.to(DEV))
            c.out.fill_(77.0)
            c.lse.fill_(77.0)
            graph.replay()
        torch.cuda.synchronize()
        for c in (a, b):
            c.check()
