"""pbd_tree_commit_served: sequences whose rows a plan gave no slots keep their cache, pages and lengths; and the packed
operators together, as a program that leaves every size on the device runs them, eagerly and as a graph."""
import math

import pytest
import torch

import paged_ref as ref
import rows_ref as rr
from paper_2607_12422_amd import binding as pbd
from test_gpu_paged_append import rope_table
from test_gpu_tree_commit import BF, DEV, F32, Commit, i32

pytestmark = pytest.mark.gpu


def served(c, before, lens=None, parents=None, starts=None):
    flat = ([p for t in (parents or c.trees) for p in t] + [0] * c.R)[: c.R]
    pbd.pbd_tree_commit_served(c.pages, i32(starts or c.starts), i32(before), i32(lens or c.lens), i32(flat), i32(c.tokens),
                               i32(c.verify), c.path, c.n, c.out, c.new, anchor=c.anchor)
    torch.cuda.synchronize()


def check(c, kept, before):
    """As c.check, with the outputs of the sequences `kept` those of skipped ones: the lengths they had."""
    for b in kept:
        assert torch.all(c.path[b] == -1) and torch.all(c.out[b] == -1)
        assert int(c.n[b]) == -1 and int(c.new[b]) == before[b] and int(c.anchor[b]) == -77
        for o in (c.path, c.out, c.n, c.new):
            o[b] = -77
    c.check(skip=kept)


def trees(sizes, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [rr.random_tree(n, g) for n in sizes]


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
def test_sequences_that_were_not_served_keep_all_they_have(dtype, D):
    sizes = [9, 12, 1, 64, 0, 17]
    lens = [30, 40, 50, 64, 20, 17]
    base = [m - n for m, n in zip(lens, sizes)]
    c = Commit(lens, trees(sizes), 2, D, dtype, right=1.0)
    served(c, base)
    check(c, (4,), base)
    assert int(c.status) == 0
    # 1, 2, 3 and 5: the length has not grown, their rows are there
    c = Commit(lens, trees(sizes), 2, D, dtype, right=1.0)
    before = [base[0], 40, 50, 64, 20, 17]
    served(c, before)
    check(c, (1, 2, 3, 4, 5), before)
    assert int(c.status) == 0


def test_fewer_slots_than_rows_and_lengths_out_of_range():
    lens, sizes = [30, 40, 50], [9, 12, 7]
    # a sequence with fewer slots than rows, not served: nothing wrong with it
    c = Commit(lens, trees(sizes), 2, 64, BF, right=1.0)
    served(c, [21, 5, 43], lens=[30, 5, 50])
    check(c, (1,), [21, 5, 43])
    assert int(c.status) == 0
    # lengths that no cache has, and slots before the first
    for length, before in ((-5, -17), (-5, -5), (5, -7), (10 ** 6, 10 ** 6 - 12), (10 ** 6, 10 ** 6), (-2 ** 31, 2 ** 31 - 12)):
        c = Commit(lens, trees(sizes), 2, 64, BF, right=1.0)
        served(c, [21, before, 43], lens=[30, length, 50])
        check(c, (1,), [21, before, 43])
        assert int(c.status) == pbd.PBD_STATUS_CAPACITY


def test_other_commits_that_are_skipped():
    lens, sizes = [30, 40, 50], [9, 12, 7]
    base = [21, 28, 43]
    for bad in (12, 5, -2, 2 ** 31 - 1):
        c = Commit(lens, trees(sizes), 2, 64, BF)
        t = list(c.trees[1])
        t[5] = bad
        served(c, base, parents=[c.trees[0], t, c.trees[2]])
        check(c, (1,), base)
        assert int(c.status) == pbd.PBD_STATUS_TREE
    c = Commit(lens, trees(sizes), 2, 64, BF)
    t = c.table.clone()
    t[1, 2] = -1
    c.pages = pbd.make_pages(c.k, c.v, t.to(DEV), n_q_heads=2, head_dim=64, status=c.status)
    served(c, base)
    check(c, (1,), base)
    assert int(c.status) == pbd.PBD_STATUS_PAGE
    c = Commit(lens, trees(sizes), 2, 64, BF)
    c.width = 9
    c.path, c.out = c.path[:, :9].contiguous(), c.out[:, :9].contiguous()
    served(c, base)
    check(c, (1,), base)
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY


class Server:
    """Four requests over a pool of a few pages, a step of which is a plan, a layout, appends and attentions of all
    layers, a commit and a release."""
    B, H, G, D, L, P, W, POOL = 4, 2, 2, 64, 3, 16, 8, 13

    def __init__(self, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.HQ, self.start = dtype, self.H * self.G, [30, 45, 20, 33]
        self.R = 90
        self.k, self.v = (torch.randn(self.L, self.POOL, self.H, self.P * self.D, generator=g).to(dtype).to(DEV) for _ in range(2))
        have = [-(-m // self.P) for m in self.start]
        ids = torch.randperm(self.POOL, generator=g).tolist()
        table = [[ids.pop() if p < h else -1 for p in range(self.W)] for h in have]
        self.free = i32(ids + [-1] * (self.POOL - len(ids)))
        self.table, self.seq_pages, self.n_free = i32(table), i32(have), i32([len(ids)])
        self.lens, self.anchor = i32(self.start), i32([-77] * self.B)
        self.status = i32([0])
        self.pages = pbd.make_pages(self.k, self.v, self.table, n_q_heads=self.HQ, head_dim=self.D, status=self.status)
        self.layers = [pbd.layer_pages(self.pages, i) for i in range(self.L)]
        self.rope = rope_table(300, self.D).to(DEV)
        B, R = self.B, self.R
        self.counts, self.parent, self.tokens, self.verify = i32([0] * B), i32([0] * R), i32([0] * R), i32([0] * R)
        self.x = torch.zeros(self.L, R, (self.HQ + 2 * self.H) * self.D, device=DEV)
        self.row_start, self.new_lens, self.after, self.n_acc = i32([0] * (B + 1)), i32([0] * B), i32([0] * B), i32([0] * B)
        self.row_seq, self.row_pos, self.slot_map = i32([0] * R), i32([0] * R), i32([0] * R)
        self.path, self.said = i32([[0] * 64] * B), i32([[0] * 64] * B)
        self.mask = torch.zeros(R, dtype=torch.int64, device=DEV)
        self.q_out = torch.zeros(self.L, R, self.HQ * self.D, dtype=dtype, device=DEV)
        self.out = torch.zeros(self.L, R, self.HQ, self.D, dtype=dtype, device=DEV)
        n = pbd.pbd_tree_attention_workspace_bytes(self.layers[0], B, R, self.W * self.P)
        self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)

    def feed(self, counts, ts, seed):
        """The inputs of a step, in place."""
        g = torch.Generator().manual_seed(seed)
        flat = [p for t in ts for p in t]
        self.counts.copy_(i32(counts))
        self.parent.copy_(i32(flat + [0] * (self.R - len(flat))))
        self.x.copy_(torch.randn(self.x.shape, generator=g).to(DEV))
        for t in (self.tokens, self.verify):
            t.copy_(torch.randint(0, 3, (self.R,), generator=g).to(torch.int32).to(DEV))

    def step(self):
        HQ, H, D = self.HQ, self.H, self.D
        pbd.pbd_page_plan(self.table, self.seq_pages, self.free, self.n_free, self.lens, self.counts, self.P, self.row_start,
                          self.row_seq, self.slot_map, self.new_lens, pos=self.lens, row_pos=self.row_pos, status=self.status)
        pbd.pbd_tree_layout(self.row_start, self.parent, self.mask, pos=self.lens, row_pos=self.row_pos, status=self.status)
        for i, one in enumerate(self.layers):
            x = self.x[i]
            pbd.pbd_paged_append_rows(one, x[:, HQ * D: (HQ + H) * D], x[:, (HQ + H) * D:], self.slot_map, self.row_pos,
                                      self.rope, q=x[:, : HQ * D], q_out=self.q_out[i])
            pbd.pbd_tree_attention(one, self.q_out[i].view(self.R, HQ, D), self.row_start, self.new_lens, self.mask,
                                   self.W * self.P, self.out[i], self.ws)
        pbd.pbd_tree_commit_served(self.pages, self.row_start, self.lens, self.new_lens, self.parent, self.tokens, self.verify,
                                   self.path, self.n_acc, self.said, self.after, anchor=self.anchor)
        pbd.pbd_page_release(self.table, self.seq_pages, self.free, self.n_free, self.after, self.P, status=self.status)

    def tensors(self):
        return {n: t for n, t in vars(self).items() if isinstance(t, torch.Tensor) and n != "ws"}

    def cached(self, b, n):
        """K and V of the first n slots of sequence b in all layers."""
        s = torch.arange(n)
        mk, mv = ref.block_maps(self.D, 8 if self.dtype == BF else 4)
        page, at = self.table[b].cpu().long()[s // self.P], (s % self.P // 16 * (16 * self.D))[:, None]
        return [torch.stack([pool.cpu()[:, page[:, None], h, at + m[s % 16]] for h in range(self.H)])
                for pool, m in ((self.k, mk), (self.v, mv))]


# rows of a step: pages for all of them; for the second not (its five are more than are free), the third needs none; none
STEPS = [[9, 3, 5, 2], [9, 64, 5, 1], [0, 30, 0, 0], [17, 64, 3, 1], [2, 1, 1, 1]]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_pool_that_runs_out(dtype):
    s = Server(dtype)
    lens, starved, anchors = list(s.start), 0, [-77] * s.B
    for turn, counts in enumerate(STEPS):
        ts = trees(counts, seed=turn)
        s.feed(counts, ts, turn)
        old = [s.cached(b, m) for b, m in enumerate(lens)]
        free, pages = int(s.n_free), s.seq_pages.tolist()
        s.status.zero_()
        s.step()
        torch.cuda.synchronize()
        asked, starts = 0, rr.starts(counts)
        missed = False
        for b, n in enumerate(counts):
            need = max(0, -(-(lens[b] + n) // s.P) - pages[b])
            asked += need
            fits = need == 0 or asked <= free
            missed |= not fits
            if n == 0 or not fits:
                starved += not fits
                assert int(s.after[b]) == lens[b] and int(s.n_acc[b]) == -1 and int(s.anchor[b]) == anchors[b]
                assert torch.all(s.path[b] == -1) and torch.all(s.said[b] == -1)
                keep = lens[b]
            else:
                rows = slice(starts[b], starts[b] + n)
                verify = s.verify[rows].tolist()
                way = rr.walk(ts[b], s.tokens[rows].tolist(), verify)
                assert s.path[b, : len(way)].tolist() == way and int(s.after[b]) == lens[b] + len(way)
                assert int(s.n_acc[b]) == len(way) - 1 and int(s.anchor[b]) == verify[way[-1]]
                keep, anchors[b] = lens[b] + len(way), verify[way[-1]]
            # what was committed before is there, bit for bit
            for got, want in zip(s.cached(b, lens[b]), old[b]):
                assert torch.equal(got, want), (turn, b)
            assert int(s.seq_pages[b]) == -(-keep // s.P)
            lens[b] = keep
        assert int(s.status) == (pbd.PBD_STATUS_CAPACITY if missed else 0)
        assert int(s.n_free) == s.POOL - sum(s.seq_pages.tolist())
        ids = [x for row in s.table.tolist() for x in row if x >= 0] + s.free[: int(s.n_free)].tolist()
        assert sorted(ids) == list(range(s.POOL))
        s.lens.copy_(s.after)
    assert starved >= 2


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_operators_together_as_a_graph(dtype):
    """A step captured once and replayed with other inputs in place, beside the same steps made eagerly: every output and
    every buffer of the two agree in every bit after every replay, eager work and synchronizations between them."""
    a, b = Server(dtype, seed=1), Server(dtype, seed=1)
    warm = Server(dtype, seed=1)
    warm.feed(STEPS[0], trees(STEPS[0]), 0)
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for turn, counts in enumerate(STEPS):
        for s in (a, b):
            s.feed(counts, trees(counts, seed=turn), turn)
        a.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        others = b.tensors()
        for name, t in a.tensors().items():
            x, y = t.contiguous().view(torch.uint8), others[name].contiguous().view(torch.uint8)
            assert torch.equal(x, y), (turn, name)
        for s in (a, b):
            s.lens.copy_(s.after)
    assert min(a.lens.tolist()) > 0 and math.isfinite(float(a.out.float().abs().sum()))
