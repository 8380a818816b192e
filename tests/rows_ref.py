"""Plain 64-bit forms of the operators on packed rows over a paged cache, shared by their tests."""
import math

import torch

from paged_ref import U


def starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return s


def causal(n, length):
    """[n][length]: row i sees the slots up to length - n + i."""
    return torch.arange(length)[None, :] <= length - n + torch.arange(n)[:, None]


def by_mask(masks, length):
    """[n][length] of a tree's rows from their masks (Python integers)."""
    n = len(masks)
    see = torch.zeros(n, length, dtype=torch.bool)
    see[:, : length - n] = True
    for i, m in enumerate(masks):
        for j in range(n):
            see[i, length - n + j] = bool(m >> j & 1)
    return see


def attention(cache, b, q, see, scale):
    """out [n][HQ][D], lse [n][HQ] of sequence b's rows q [n][HQ][D], and the bounds of their errors.

    scores: fp32 sums of products of exact operands, D + 4 roundings of partial sums: ds = (D + 4) U scale max sum |q k|.
    weights: 2 ds from the score and the maximum or sum it is set against; 3 roundings of the score in log2 units
      (scale, product, difference), of which the difference's argument is at most twice the largest score; 4 U from the exponential.  A weight that meets the values is rounded to the cache's type.
    sums: len + 80 roundings of partial sums below sum w |v|, of tiles, waves and splits.
    the output is rounded to the cache's type once."""
    n, HQ, D = q.shape
    length = see.shape[1]
    H = cache.H
    G = HQ // H
    half = torch.finfo(cache.dtype).eps / 2 if cache.dtype == torch.bfloat16 else 0.0
    k, v = cache.dk[b, :, :length].double(), cache.dv[b, :, :length].double()
    x = q.double().view(n, H, G, D).permute(1, 2, 0, 3)
    s = torch.matmul(x, k[:, None].transpose(2, 3)) * scale                       # [H][G][n][len]
    size = torch.matmul(x.abs(), k[:, None].abs().transpose(2, 3)) * scale
    size = torch.where(see, size, 0.0).amax(-1)
    s = torch.where(see, s, -math.inf)
    ds = (D + 4) * U * size
    lse = torch.logsumexp(s, -1)
    none = ~see.any(-1)
    w = torch.where(see, torch.exp(s - lse[..., None]), 0.0)
    w[..., none, :] = 0.0
    vv = v[:, None]
    out, mass = torch.matmul(w, vv), torch.matmul(w, vv.abs())
    rel = 2 * ds + 3 * U * 3 * size + (length + 80 + 8) * U
    tol = mass * (rel[..., None] + half * 1.01) + out.abs() * (torch.finfo(cache.dtype).eps / 2) * 1.01 + 1e-30
    # (slots that are not seen may hold anything: `out` is for finite values)
    back = lambda t: t.permute(2, 0, 1, 3).reshape(n, HQ, D)
    flat = lambda t: t.permute(2, 0, 1).reshape(n, HQ)
    lse_tol = ds + 9 * U * size + (length + 88) * U + 4 * U * torch.where(none, 0.0, lse.abs())
    return back(out), flat(lse), back(tol), flat(lse_tol)


def ancestors(parents):
    masks = []
    for i, p in enumerate(parents):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    return masks


def random_tree(n, g, back=4):
    return [-1] + [max(0, i - 1 - int(torch.randint(0, back, (1,), generator=g))) for i in range(1, n)] if n else []


def to_i64(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64)


def walk(parents, tokens, verify):
    path = [0]
    while True:
        fit = [i for i in range(1, len(parents)) if parents[i] == path[-1] and tokens[i] == verify[path[-1]]]
        if not fit:
            return path
        path.append(fit[0])


class Tables:
    """Tables, counts and stack of free pages, and what a plan or a release makes of them."""

    def __init__(self, table, seq_pages, free, n_free, page):
        self.table, self.seq_pages, self.free, self.n_free, self.page = table, seq_pages, free, n_free, page

    def plan(self, lens, new, pos, max_rows):
        B, W, P, N = len(lens), len(self.table[0]), self.page, len(self.free)
        r = dict(row_start=[0], row_seq=[-1] * max_rows, row_pos=[0] * max_rows, slot_map=[-1] * max_rows,
                 new_lens=list(lens), status=0)
        f = self.n_free
        if f < 0 or f > N:
            r["status"] |= 1
            f = 0
        jobs, rows, want = [], 0, 0
        for b in range(B):
            m, n, h = lens[b], new[b], self.seq_pages[b]
            rows += max(0, n)
            ok = m >= 0 and n >= 0 and 0 <= h <= W and m <= h * P and m + n <= W * P and rows <= max_rows
            need = max(0, -(-(m + n) // P) - h) if ok else 0
            want += need
            jobs.append((ok, need, want, rows))
        taken = max([w for ok, need, w, _ in jobs if need and w <= f], default=0)
        if any(not 0 <= self.free[f - 1 - i] < N for i in range(taken)):
            r["status"] |= 16
            f = taken = 0
        for b, (ok, need, upto, end) in enumerate(jobs):
            first = end - max(0, new[b])
            r["row_start"][b:] = [min(first, max_rows), min(end, max_rows)]
            served = ok and (need == 0 or upto <= f)
            if served:
                for i in range(need):
                    self.table[b][self.seq_pages[b] + i] = self.free[f - 1 - (upto - need + i)]
                self.seq_pages[b] += need
                r["new_lens"][b] = lens[b] + new[b]
            else:
                r["status"] |= 1
            for i in range(first, min(end, max_rows)):
                s = lens[b] + i - first
                r["row_seq"][i] = b
                r["row_pos"][i] = pos[b] + i - first
                if served:
                    r["slot_map"][i] = self.table[b][s // P] * P + s % P
        if taken:
            self.n_free = f - taken
        return r

    def release(self, keep):
        B, W, P, N = len(keep), len(self.table[0]), self.page, len(self.free)
        status, back = 0, []
        for b in range(B):
            h, k = self.seq_pages[b], keep[b]
            if not 0 <= h <= W or k < 0:
                status |= 1
                continue
            ids = [(b, p) for p in range(min(h, -(-k // P)), h)]
            if any(not 0 <= self.table[b][p] < N for _, p in ids):
                status |= 16
                continue
            back += ids
        if self.n_free < 0 or self.n_free + len(back) > N:
            return status | 1
        for b, p in reversed(back):
            self.free[self.n_free] = self.table[b][p]
            self.n_free += 1
            self.table[b][p] = -1
            self.seq_pages[b] -= 1
        return status
