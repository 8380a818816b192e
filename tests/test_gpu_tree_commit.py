"""pbd_tree_layout and pbd_tree_commit against plain forms: trees of every size, paths of every kind, all layers, and what
must stay as it was; and the packed operators together, as a server would use them."""
import math

import pytest
import torch

import paged_ref as ref
import rows_ref as rr
from paper_2607_12422_amd import binding as pbd
from test_gpu_paged_append import rope_table

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def layout(trees, pos=None, rows=None, starts=None):
    starts = starts or rr.starts([len(t) for t in trees])
    R = rows or max(1, starts[-1])
    flat = ([p for t in trees for p in t] + [0] * R)[:R]
    mask = torch.full((R,), -77, dtype=torch.int64, device=DEV)
    row_pos = torch.full((R,), -77, dtype=torch.int32, device=DEV) if pos else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    pbd.pbd_tree_layout(i32(starts), i32(flat), mask, pos=i32(pos) if pos else None, row_pos=row_pos, status=status)
    return mask.cpu(), row_pos.cpu() if pos else None, int(status)


@pytest.mark.parametrize("with_pos", [False, True])
def test_layouts(with_pos):
    g = torch.Generator().manual_seed(2)
    sizes = [0, 1, 2, 17, 63, 64, 64, 5]
    trees = [rr.random_tree(n, g) for n in sizes]
    trees[6] = list(range(-1, 63))                   # one line of 64
    trees[7] = [-1, -1, 0, 1, -1]                    # several roots
    pos = [10 * b for b in range(len(trees))] if with_pos else None
    mask, at, status = layout(trees, pos, rows=sum(map(len, trees)) + 9)
    want = [m for t in trees for m in rr.ancestors(t)]
    assert status == 0 and torch.equal(mask[: len(want)], rr.to_i64(want)) and torch.all(mask[len(want):] == -77)
    if with_pos:
        depth = [10 * b + bin(m).count("1") - 1 for b, t in enumerate(trees) for m in rr.ancestors(t)]
        assert at[: len(want)].tolist() == depth and torch.all(at[len(want):] == -77)


def test_layouts_that_are_skipped():
    good = [-1, 0, 1]
    for bad in ([-1, 1], [-1, 0, 5], [0, 0], [-2, 0], [-1, 2 ** 31 - 1], [-1, -2 ** 31]):
        mask, _, status = layout([good, bad, good])
        assert status == pbd.PBD_STATUS_TREE
        n = len(bad)
        assert torch.all(mask[3: 3 + n] == -77) and mask[:3].tolist() == mask[3 + n:].tolist() == [1, 3, 7]
    mask, _, status = layout([good, [-1] * 65, good])
    assert status == pbd.PBD_STATUS_CAPACITY and torch.all(mask[3:68] == -77) and mask[68:].tolist() == [1, 3, 7]
    for starts in ([0, 3, 7], [0, 3, 2], [-1, 3, 6]):
        mask, _, status = layout([good, good], rows=6, starts=starts)
        assert status == pbd.PBD_STATUS_CAPACITY


class Commit:
    """Trees at the end of sequences over a cache of several layers; verify tokens that follow `follow` of each path."""

    def __init__(self, lens, trees, H, D, dtype, layers=2, page=16, major="page", seed=0, vocab=4, extra=0, right=0.8):
        g = torch.Generator().manual_seed(seed)
        self.trees, self.lens, self.dtype = trees, lens, dtype
        self.caches = [ref.Cache(lens, H, D, dtype, page=page, major=major, seed=seed + 100 * i) for i in range(layers)]
        for c in self.caches[1:]:
            c.table = self.caches[0].table
            for pool in (c.k, c.v):
                pool.fill_(math.nan)
            for b, m in enumerate(lens):
                c.put(b, 0, c.dk[b, :, :m], c.dv[b, :, :m])
        self.starts = rr.starts([len(t) for t in trees])
        self.R = max(1, self.starts[-1] + extra)
        self.tokens = torch.randint(0, vocab, (self.R,), generator=g).tolist()
        self.verify = torch.randint(0, vocab, (self.R,), generator=g).tolist()
        for b, t in enumerate(trees):
            for i in range(len(t)):
                kids = [j for j in range(len(t)) if t[j] == i]
                if kids and float(torch.rand(1, generator=g)) < right:
                    pick = kids[int(torch.randint(0, len(kids), (1,), generator=g))]
                    self.verify[self.starts[b] + i] = self.tokens[self.starts[b] + pick]
        stack = lambda ts: torch.stack([t.permute(1, 0, 2) if major == "head" else t for t in ts]).to(DEV)
        k, v = stack([c.k for c in self.caches]), stack([c.v for c in self.caches])
        if major == "head":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        self.k, self.v = k, v
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.table = self.caches[0].table.clone()
        self.pages = pbd.make_pages(k, v, self.table.to(DEV), n_q_heads=H, head_dim=D, status=self.status)
        self.width = max(map(len, trees), default=1) + 2
        B = len(trees)
        full = lambda *s: torch.full(s, -77, dtype=torch.int32, device=DEV)
        self.path, self.out, self.n, self.new, self.anchor = full(B, self.width), full(B, self.width), full(B), full(B), full(B)

    def run(self, lens=None, parents=None, starts=None):
        flat = ([p for t in (parents or self.trees) for p in t] + [0] * self.R)[: self.R]
        pbd.pbd_tree_commit(self.pages, i32(starts or self.starts), i32(lens or self.lens), i32(flat), i32(self.tokens),
                            i32(self.verify), self.path, self.n, self.out, self.new, anchor=self.anchor)
        torch.cuda.synchronize()

    def check(self, skip=()):
        k, v = self.k.cpu(), self.v.cpu()
        for b, t in enumerate(self.trees):
            if b in skip or not t:
                for o in (self.path, self.out, self.n, self.new, self.anchor):
                    assert torch.all(o[b] == -77)
                path = []
            else:
                s = self.starts[b]
                tok, ver = self.tokens[s: s + len(t)], self.verify[s: s + len(t)]
                path = rr.walk(t, tok, ver)
                fill = [-1] * (self.width - len(path))
                assert self.path[b].tolist() == path + fill
                assert self.out[b].tolist() == [tok[i] for i in path[1:]] + [ver[path[-1]]] + fill
                assert int(self.n[b]) == len(path) - 1 and int(self.anchor[b]) == ver[path[-1]]
                assert int(self.new[b]) == self.lens[b] - len(t) + len(path)
            base = self.lens[b] - len(t)
            for layer, c in enumerate(self.caches):
                gk, gv = c.get(b, self.lens[b], k[layer], v[layer])
                wk, wv = c.dk[b, :, : self.lens[b]].clone(), c.dv[b, :, : self.lens[b]].clone()
                for i, p in enumerate(path):
                    wk[:, base + i], wv[:, base + i] = c.dk[b, :, base + p], c.dv[b, :, base + p]
                assert torch.equal(gk, wk) and torch.equal(gv, wv), (b, layer)
        # nothing past the sequences
        for layer, c in enumerate(self.caches):
            used = torch.zeros(k.shape[1], dtype=torch.bool)
            for b, m in enumerate(self.lens):
                used[c.table[b, : -(-m // c.page)].long()] = True
            assert torch.isnan(k[layer][~used]).all() and torch.isnan(v[layer][~used]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("right", [0.0, 0.8, 1.0])
def test_paths(dtype, D, right):
    g = torch.Generator().manual_seed(D)
    sizes = [(1, 1), (64, 64), (70, 64), (17, 17), (33, 20), (200, 63), (40, 0), (31, 2)]
    trees = [rr.random_tree(n, g) for _, n in sizes]
    c = Commit([m for m, _ in sizes], trees, 2, D, dtype, seed=D, right=right, extra=5)
    c.run()
    c.check()
    assert int(c.status) == 0


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("major", ["page", "head"])
def test_pages_layers_and_strides(page, major):
    g = torch.Generator().manual_seed(page)
    c = Commit([100, 77, 64, 130], [rr.random_tree(n, g, back=2) for n in (40, 17, 64, 64)], 3, 64, BF, layers=3, page=page,
               major=major, seed=page, right=1.0)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_layers_of_many_trees(dtype):
    """More layers of sequences' heads than run at once, in a number that four does not divide."""
    g = torch.Generator().manual_seed(7)
    sizes = [3 + b % 30 for b in range(60)]
    c = Commit([n + b % 7 for b, n in enumerate(sizes)], [rr.random_tree(n, g, back=2) for n in sizes], 5, 64, dtype, layers=7,
               seed=4, right=1.0)
    c.run()
    c.check()


def test_a_line_of_64_and_a_path_of_the_last_ones():
    line = list(range(-1, 63))
    late = [-1] * 32 + [0] + list(range(32, 63))     # node 32 hangs on node 0, then a line
    for dtype in (BF, F32):
        c = Commit([64, 100], [line, late], 2, 128, dtype, right=1.0, vocab=1000)
        c.run()
        c.check()
        assert c.n.tolist() == [63, 32]


def test_equal_tokens_go_to_the_lowest_child():
    c = Commit([20], [[-1, 0, 0, 1, 2, 2]], 1, 64, BF, vocab=1)
    c.run()
    c.check()
    assert c.path[0, :3].tolist() == [0, 1, 3]


def test_one_layer_and_no_anchor():
    c = Commit([20], [[-1, 0, 0, 1, 2, 2]], 2, 64, BF, layers=1, vocab=2)
    pages = pbd.layer_pages(c.pages, 0)
    pbd.pbd_tree_commit(pages, i32(c.starts), i32(c.lens), i32(c.trees[0]), i32(c.tokens), i32(c.verify), c.path, c.n, c.out, c.new)
    assert int(c.anchor) == -77
    c.anchor.fill_(c.verify[int(c.path[0, int(c.n[0])])])
    c.check()


def test_commits_that_are_skipped():
    g = torch.Generator().manual_seed(1)
    trees = [rr.random_tree(n, g) for n in (9, 12, 7)]
    lens = [30, 40, 50]
    for kw in (dict(lens=[30, 11, 50]), dict(lens=[30, -5, 50]), dict(lens=[30, 10 ** 6, 50])):
        c = Commit(lens, trees, 2, 64, BF)
        c.run(**kw)
        c.check(skip=(1,))
        assert int(c.status) == pbd.PBD_STATUS_CAPACITY
    for bad in (12, 5, -2, 2 ** 31 - 1):
        c = Commit(lens, trees, 2, 64, BF)
        t = list(trees[1])
        t[5] = bad
        c.run(parents=[trees[0], t, trees[2]])
        c.check(skip=(1,))
        assert int(c.status) == pbd.PBD_STATUS_TREE
    for bad in (-1, 2 ** 31 - 1):
        c = Commit(lens, trees, 2, 64, BF)
        t = c.table.clone()
        t[1, 2] = bad
        c.pages = pbd.make_pages(c.k, c.v, t.to(DEV), n_q_heads=2, head_dim=64, status=c.status)
        c.run()
        c.check(skip=(1,))
        assert int(c.status) == pbd.PBD_STATUS_PAGE
    # a tree that does not fit the outputs
    c = Commit(lens, trees, 2, 64, BF)
    c.width = 9
    c.path, c.out = c.path[:, :9].contiguous(), c.out[:, :9].contiguous()
    c.run()
    c.check(skip=(1,))
    assert int(c.status) == pbd.PBD_STATUS_CAPACITY


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_operators_together(dtype):
    """Prompts of several requests, then two rounds of trees: pages, rows, attention, acceptance; against a server that keeps
    dense caches.  The second round runs as a graph would: every size on the device."""
    g = torch.Generator().manual_seed(9)
    B, H, G, D, page, L = 3, 2, 2, 64, 16, 2
    HQ, esz = H * G, torch.finfo(dtype).eps / 2
    pool = 40
    k = torch.full((L, pool, H, page * D), math.nan, dtype=dtype, device=DEV)
    v = k.clone()
    table = torch.full((B, 12), -1, dtype=torch.int32, device=DEV)
    seq_pages, n_free = i32([0] * B), i32([pool])
    free = torch.randperm(pool, generator=g).to(torch.int32).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    pages = pbd.make_pages(k, v, table, n_q_heads=HQ, head_dim=D, status=status)
    rope = rope_table(300, D)
    drope = rope.to(DEV)
    lens = i32([0] * B)
    dense = [[[torch.zeros(H, 0, D) for _ in range(2)] for _ in range(L)] for _ in range(B)]   # [seq][layer][k, v]
    kept = [0] * B
    for turn, counts in enumerate(([37, 1, 90], [9, 30, 17], [64, 2, 33])):
        tree = turn > 0
        R = sum(counts) + 4
        starts = rr.starts(counts)
        trees = [rr.random_tree(n, g) for n in counts]
        row_start, row_seq, row_pos, slot_map, new_lens = i32([0] * (B + 1)), i32([0] * R), i32([0] * R), i32([0] * R), i32([0] * B)
        pbd.pbd_page_plan(table, seq_pages, free, n_free, lens, i32(counts), page, row_start, row_seq, slot_map, new_lens,
                          pos=lens, row_pos=row_pos, status=status)
        parent = i32([p for t in trees for p in t] + [0] * 4)
        mask = torch.zeros(R, dtype=torch.int64, device=DEV)
        if tree:
            pbd.pbd_tree_layout(row_start, parent, mask, pos=lens, row_pos=row_pos, status=status)
        at = row_pos.cpu()
        for layer in range(L):
            x = torch.randn(R, (HQ + 2 * H) * D, generator=g)
            dx = x.to(DEV)
            q_out = torch.zeros(R, HQ * D, dtype=dtype, device=DEV)
            one = pbd.layer_pages(pages, layer)
            pbd.pbd_paged_append_rows(one, dx[:, HQ * D: (HQ + H) * D], dx[:, (HQ + H) * D:], slot_map, row_pos, drope,
                                      q=dx[:, : HQ * D], q_out=q_out)
            out = torch.full((R, HQ, D), 77.0, dtype=dtype, device=DEV)
            q = q_out.view(R, HQ, D)
            if tree:
                ws = torch.empty(pbd.pbd_tree_attention_workspace_bytes(one, B, R, 192), dtype=torch.uint8, device=DEV)
                pbd.pbd_tree_attention(one, q, row_start, new_lens, mask, 192, out, ws)
            else:
                ws = torch.empty(pbd.pbd_packed_attention_workspace_bytes(one, B, R, 192), dtype=torch.uint8, device=DEV)
                pbd.pbd_packed_attention(one, q, row_start, new_lens, 192, out, ws)
            out = out.double().cpu()
            half = D // 2

            def turned(y, pos):
                a, b = y.double()[..., :half], y.double()[..., half:]
                c, s = rope[pos][:, None, :, 0].double(), rope[pos][:, None, :, 1].double()
                return torch.cat((a * c - b * s, b * c + a * s), -1)

            for b, n in enumerate(counts):
                rows = slice(starts[b], starts[b] + n)
                where = at[rows].long()
                depth = [bin(m).count("1") - 1 for m in rr.ancestors(trees[b])]
                assert where.tolist() == [kept[b] + (depth[i] if tree else i) for i in range(n)]
                nk = turned(x[rows, HQ * D: (HQ + H) * D].unflatten(1, (H, D)), where).to(dtype).transpose(0, 1)
                nv = x[rows, (HQ + H) * D:].unflatten(1, (H, D)).to(dtype).transpose(0, 1)
                old = dense[b][layer]
                old[0], old[1] = torch.cat((old[0], nk.double()), 1), torch.cat((old[1], nv.double()), 1)
                length = old[0].shape[1]
                see = rr.by_mask(rr.ancestors(trees[b]), length) if tree else rr.causal(n, length)
                c = type("C", (), dict(H=H, dtype=dtype, dk=old[0][None], dv=old[1][None]))
                rq = turned(x[rows, : HQ * D].unflatten(1, (HQ, D)), where).to(dtype)
                want, _, tol, _ = rr.attention(c, 0, rq, see, D ** -0.5)
                # a rounding of a key or query may fall to the other side: scores differ by one step of one element's product,
                # less than 2 eps (|q| |k|) / sqrt(D) in all, the weights by twice that
                size = rq.double().norm(dim=-1).max() * old[0].norm(dim=-1).max() * D ** -0.5
                slip = 4 * 2 * esz * size if dtype == BF else 64 * ref.U * size
                assert torch.all((out[rows] - want).abs() <= tol + slip * old[1].abs().max()), (turn, layer, b)
            assert torch.all(out[starts[-1]:] == 77.0)
        if not tree:
            lens = new_lens.clone()
            kept = list(counts)
            continue
        tokens = torch.randint(0, 3, (R,), generator=g)
        verify = torch.randint(0, 3, (R,), generator=g)
        path, said = i32([[0] * 64] * B), i32([[0] * 64] * B)
        n_acc, after = i32([0] * B), i32([0] * B)
        pbd.pbd_tree_commit(pages, row_start, new_lens, parent, tokens.to(torch.int32).to(DEV), verify.to(torch.int32).to(DEV),
                            path, n_acc, said, after)
        pbd.pbd_page_release(table, seq_pages, free, n_free, after, page, status=status)
        for b, n in enumerate(counts):
            way = rr.walk(trees[b], tokens[starts[b]:starts[b] + n].tolist(), verify[starts[b]:starts[b] + n].tolist())
            assert path[b, : len(way)].tolist() == way and int(after[b]) == kept[b] + len(way)
            for layer in range(L):
                for i in range(2):
                    old = dense[b][layer][i]
                    dense[b][layer][i] = torch.cat((old[:, : kept[b]], old[:, [kept[b] + w for w in way]]), 1)
            kept[b] += len(way)
        assert seq_pages.tolist() == [-(-m // page) for m in kept]
        assert int(n_free) == pool - sum(seq_pages.tolist())
        lens = after.clone()
    assert int(status) == 0
