"""Plain 64-bit forms of the paged-cache operators and the layout of the cache,
shared by their tests."""
import math

import torch

U = 2.0 ** -24          # half a step of fp32


def kv_index(slot, dim, E):
    """Element of (slot, dim) inside a 16-slot block: of K, of V (include/pbd.h)."""
    return ((dim // E) * 16 + slot) * E + dim % E, ((dim // 16 * 4 + slot // 4) * 16 + dim % 16) * 4 + slot % 4


def block_maps(D, E):
    s, d = torch.arange(16)[:, None], torch.arange(D)[None, :]
    return kv_index(s, d, E)


class Cache:
    """A paged cache of B sequences of lens slots: dense K and V float64 [B][H][cap][D] (the values the pool
    holds), the pool around them filled with NaN, its pages anywhere."""

    def __init__(self, lens, H, D, dtype, page=16, major="page", spare=3, seed=0, room=0, device="cpu"):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H, self.D, self.page, self.dtype = list(lens), H, D, page, dtype
        B = len(self.lens)
        self.E = 16 // torch.empty(0, dtype=dtype).element_size()
        self.width = max(1, -(-(max(self.lens) + room) // page))
        n = B * self.width + spare
        shape = (H, n, page * D) if major == "head" else (n, H, page * D)
        self.k, self.v = (torch.full(shape, math.nan, dtype=dtype) for _ in range(2))
        if major == "head":
            self.k, self.v = self.k.permute(1, 0, 2), self.v.permute(1, 0, 2)
        self.table = torch.randperm(n, generator=g)[: B * self.width].to(torch.int32).view(B, self.width)
        cap = self.width * page
        self.dk, self.dv = (torch.randn(B, H, cap, D, generator=g).to(dtype) for _ in range(2))
        for b, m in enumerate(self.lens):
            self.put(b, 0, self.dk[b, :, :m], self.dv[b, :, :m])
            # pages past the ones in use: ids that must not be followed
            self.table[b, -(-(m + room) // page):] = -7
        self.device = device

    def places(self, b, slots):
        """(page, element of dim 0.. inside a head's page for K, for V) of slots."""
        mk, mv = block_maps(self.D, self.E)
        base = (slots % self.page // 16 * (16 * self.D))[:, None]
        return self.table[b].long()[slots // self.page], base + mk[slots % 16], base + mv[slots % 16]

    def put(self, b, first, k, v):
        page, ik, iv = self.places(b, torch.arange(first, first + k.shape[1]))
        for h in range(self.H):
            self.k[page[:, None], h, ik] = k[h]
            self.v[page[:, None], h, iv] = v[h]

    def get(self, b, n, k=None, v=None):
        """The first n slots of sequence b as [H][n][D], from the given pools."""
        k, v = self.k if k is None else k, self.v if v is None else v
        page, ik, iv = self.places(b, torch.arange(n))
        return (torch.stack([k[page[:, None], h, ik] for h in range(self.H)]),
                torch.stack([v[page[:, None], h, iv] for h in range(self.H)]))

    def to(self, device):
        """(k, v, table) on the device, the strides kept."""
        def move(t):
            base = t.permute(1, 0, 2) if not t.is_contiguous() else t
            moved = base.to(device)
            return moved.permute(1, 0, 2) if base is not t else moved
        return move(self.k), move(self.v), self.table.to(device)


def attention(cache, q, scale):
    """For each sequence: out [HQ][D], lse [HQ], weight sums [H][len], and the bounds of their errors in fp32
    arithmetic on the values the kernel reads.

    scores: products of exact operands (a bf16 cache: the query as three bf16 terms) summed in fp32, at most
      D + 4 roundings of partial sums below sum |q k|:  ds = (D + 4) U scale max sum |q k|.
    weights: 2 ds from the score and its maximum, 4 U from the exponential; a bf16 cache takes them as three
      bf16 terms, all of their 24 bits.
    sums: a wave adds at most 32 steps of 32 slots, four waves and the splits are joined: at most
      min(len, 1100) + 80 roundings of partial sums below sum w |v|."""
    G = q.shape[1] // cache.H
    res = []
    for b, n in enumerate(cache.lens):
        k, v = cache.dk[b, :, :n].double(), cache.dv[b, :, :n].double()
        x = q[b].double().view(cache.H, G, 1, -1)
        s = (x * k[:, None]).sum(-1) * scale                      # [H][G][n]
        size = ((x.abs() * k[:, None].abs()).sum(-1) * scale).amax(-1) if n else torch.zeros(cache.H, G)
        ds = (cache.D + 4) * U * size.double()
        depth = min(n, 1100) + 80
        lse = torch.logsumexp(s, -1) if n else torch.full((cache.H, G), -math.inf, dtype=torch.float64)
        w = torch.exp(s - lse[..., None])
        out = torch.matmul(w, v)                                  # [H][G][D]
        rel = 2 * ds + (depth + 8) * U
        tol = torch.matmul(w, v.abs()) * rel[..., None] + 1e-30
        res.append(dict(out=out.flatten(0, 1), lse=lse.flatten(), w=w.sum(1), out_tol=tol.flatten(0, 1),
                        lse_tol=(ds + (depth + 8) * U + 4 * U * lse.abs()).flatten(),
                        w_tol=(w * rel[..., None]).sum(1) + 1e-30))
    return res


def kept(score, slot_pos, n, keep, last, sink):
    """The slots of one head that stay, ascending, and its moves [(to, from)]."""
    def rank(i):
        if slot_pos is not None and (slot_pos[i] >= last or slot_pos[i] < sink):
            return (0, 0.0, i)
        return (2, 0.0, i) if math.isnan(score[i]) else (1, -score[i], i)
    keep = min(keep, n)
    stay = set(sorted(range(n), key=rank)[:keep])
    return sorted(stay), list(zip([i for i in range(keep) if i not in stay],
                                  [i for i in range(keep, n) if i in stay]))
