"""Performance cases of the paged-cache and log-probability operators on one GPU.

A program that serves with this framework one token at a time appends the new
token's keys and values to a paged cache, attends over the cache, evicts what
was attended to least once a sequence is over its budget, and reports the log
probabilities of the tokens it chose.  Each case is one such call.

A case is a dict of
  op       "attend"   attention of one new token over the cache (scored: the weights are accumulated too)
           "append"   new rows into the cache: per-head RMSNorm, RoPE, K/V to the slots after the last
           "evict"    the slots of least accumulated weight out, the others moved together
           "logprobs" log probabilities of given tokens, entropy, top alternatives
  dtype    "bf16" or "f32": the cache's (logprobs: the logits') type
  batch, lo, hi    sequences, and the range their lengths are drawn from
  hq, hkv, hd      query heads, KV heads, head size
  page, major      positions per page; "page": [page][head][...], "head": [head][page][...] (the order of
                   a context's own cache)
  rows             append: new rows per sequence at most;  logprobs: rows of logits
  keep, recent, sink   evict: slots kept, last positions and first positions that always stay
  vocab, pad, top, masked   logprobs: columns, unused columns at each row's end, alternatives, whether
                   part of the vocabulary is masked by minus infinity

Cache blocks hold 16 positions: K as [hd / E][16][E] with E = 16 bytes of elements, V as
[hd / 16][4][16][4], (dim // 16, position // 4, dim % 16, position % 4).  A page of one head is
page / 16 such blocks.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
THETA = 1e6


def listed():
    tiny = dict(dtype="f32", hq=4, hkv=2, hd=64, page=16, major="head")
    qwen = dict(dtype="bf16", hq=16, hkv=8, hd=128, page=16, major="page")
    return [
        # the tiny decoder's short sequence: latency alone
        dict(tiny, name="attend_b1_n300_f32", op="attend", batch=1, lo=300, hi=300, scored=False),
        # one user, an ordinary context
        dict(qwen, name="attend_b1_n4096", op="attend", batch=1, lo=4096, hi=4096, scored=False),
        # a serving batch of ragged lengths, eight query heads a KV head, larger pages
        dict(qwen, name="attend_b24_ragged_g8", op="attend", batch=24, lo=256, hi=4096, hq=32, hkv=4, page=64,
             scored=False),
        # the largest batch at its longest, with the weights accumulated for the eviction
        dict(qwen, name="attend_b32_n8192_scored", op="attend", batch=32, lo=8192, hi=8192, scored=True),
        # a decode step's rows
        dict(qwen, name="append_b32_r1", op="append", batch=32, lo=100, hi=400, rows=1, norm=True),
        # a prompt chunk of several users, ragged
        dict(qwen, name="append_b4_r1000", op="append", batch=4, lo=0, hi=777, rows=1000, norm=True, page=32),
        # the tiny decoder over its budget by a block
        dict(tiny, name="evict_b1_n640_f32", op="evict", batch=1, lo=640, hi=640, keep=512, recent=64, sink=4),
        # long odd lengths of few users, halved
        dict(qwen, name="evict_b2_n40001", op="evict", batch=2, lo=39000, hi=40001, keep=20000, recent=1024, sink=4,
             page=64),
        # the largest batch at its longest, halved
        dict(qwen, name="evict_b32_n8192", op="evict", batch=32, lo=8192, hi=8192, keep=4096, recent=256, sink=0,
             major="head"),
        # one decoded token of the tiny decoder
        dict(name="logprobs_r1_v4096", op="logprobs", dtype="f32", rows=1, vocab=4096, pad=0, top=5, masked=False),
        # the rows of one verify pass, with twenty alternatives
        dict(name="logprobs_r17_v151936", op="logprobs", dtype="f32", rows=17, vocab=151936, pad=0, top=20,
             masked=False),
        # the rows of the largest verify pass, logits kept in bf16
        dict(name="logprobs_r1056_bf16", op="logprobs", dtype="bf16", rows=1056, vocab=151936, pad=0, top=8,
             masked=False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "evict", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "logprobs":
        rows = _log(rng, 1, 1056)
        vocab = _log(rng, 300, 152000)
        if dtype == "f32":
            rows = min(rows, 500)
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 7, 64]),
                    top=rng.choice([0, 1, 5, 20, 32]), masked=rng.random() < 0.3)
    hkv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, dtype=dtype, hkv=hkv, hq=hkv * rng.choice([1, 2, 3, 4, 5, 8, 16]), hd=rng.choice([64, 128]),
             page=rng.choice([16, 16, 32, 64, 128]), major=rng.choice(["page", "head"]))
    most = 32 * 8192 * 8 * 128 * 2 // (hkv * c["hd"] * (2 if dtype == "bf16" else 4))
    if op == "append":
        rows = _log(rng, 1, 1024)
        hi = _log(rng, 1, 4000)
        return dict(c, batch=_log(rng, 1, max(1, min(64, 4000 // rows))), lo=rng.randint(0, hi), hi=hi, rows=rows,
                    norm=rng.random() < 0.7)
    batch = _log(rng, 1, 64)
    hi = _log(rng, 1, min(65000, most // batch))
    c.update(batch=batch, lo=rng.randint(hi // 4, hi), hi=hi)
    if op == "attend":
        return dict(c, scored=rng.random() < 0.4)
    keep = rng.randint(0, hi)
    return dict(c, keep=keep, recent=rng.randint(0, keep // 2), sink=rng.choice([0, 0, 4]))


def _generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + stream)


def _cache(case, lens, room, g):
    """(K pool, V pool, page table) for sequences of lens slots with room for `room` more; each pool
    [pages][heads][page * hd], the pages of a sequence anywhere in it."""
    dt = TYPES[case["dtype"]]
    H, n = case["hkv"], case["page"] * case["hd"]
    per = max(1, -(-(case["hi"] + room) // case["page"]))
    B = case["batch"]
    pages = B * per + 3

    def pool():
        if case["major"] == "head":
            return torch.randn(H, pages, n, generator=g, device=DEV, dtype=dt).permute(1, 0, 2)
        return torch.randn(pages, H, n, generator=g, device=DEV, dtype=dt)

    table = torch.randperm(pages, generator=g, device=DEV)[: B * per].to(torch.int32).view(B, per)
    used = (torch.arange(per, device=DEV) * case["page"])[None, :] < (lens + room)[:, None]
    return pool(), pool(), torch.where(used, table, torch.full_like(table, -1)).contiguous()


def prepare(case, seed):
    g = _generator(seed, 0)
    i32 = dict(dtype=torch.int32, device=DEV)
    f32 = dict(dtype=torch.float32, device=DEV)
    s = dict(case=case)
    if case["op"] == "logprobs":
        R, V = case["rows"], case["vocab"]
        x = torch.randn(R, V + case["pad"], generator=g, **f32) * 3.0
        if case["masked"]:
            x[:, :V] = torch.where(torch.rand(R, V, generator=g, **f32) < 0.4, -math.inf, x[:, :V])
        s["logits"] = x.to(TYPES[case["dtype"]])[:, :V]
        # chosen tokens: likely ones for the most part
        s["tokens"] = torch.where(torch.rand(R, generator=g, **f32) < 0.7, x[:, :V].argmax(-1),
                                  torch.randint(0, V, (R,), generator=g, device=DEV)).to(torch.int32)
        return s
    B, H, HQ, D = case["batch"], case["hkv"], case["hq"], case["hd"]
    lens = torch.randint(case["lo"], case["hi"] + 1, (B,), generator=g, **i32)
    room = case["rows"] if case["op"] == "append" else 0
    s["lens"] = lens
    s["k"], s["v"], s["table"] = _cache(case, lens, room, g)
    cap = s["table"].shape[1] * case["page"]
    if case["op"] == "attend":
        s["q"] = torch.randn(B, HQ, D, generator=g, **f32)
        s["score"] = torch.rand(B, H, cap, generator=g, **f32) if case["scored"] else None
        return s
    if case["op"] == "append":
        R = case["rows"]
        qkv = torch.randn(B, R, (HQ + 2 * H) * D, generator=g, **f32)
        s["qkv"] = qkv
        s["q"] = qkv[:, :, : HQ * D]
        s["new_k"] = qkv[:, :, HQ * D : (HQ + H) * D]
        s["new_v"] = qkv[:, :, (HQ + H) * D :]
        s["n_new"] = torch.randint(max(1, R // 2), R + 1, (B,), generator=g, **i32)
        s["pos"] = lens + 11
        dt = TYPES[case["dtype"]]
        for name in ("q_norm", "k_norm"):
            gain = 1.0 + 0.02 * torch.randn(D, generator=g, **f32)
            s[name] = gain.to(dt) if case["norm"] else None
        at = torch.arange(case["hi"] + 11 + R, device=DEV, dtype=torch.float64)
        ang = at[:, None] * THETA ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
        s["rope"] = torch.stack((ang.cos(), ang.sin()), -1).to(torch.float32).contiguous()
        s["q_out"] = torch.zeros(B, R, HQ * D, **f32)
        s["score"] = torch.rand(B, H, cap, generator=g, **f32)
        s["slot_pos"] = torch.full((B, H, cap), -1, **i32)
        s["len_out"] = torch.zeros(B, **i32)
        return s
    # accumulated weights: many orders of magnitude, some slots never attended to
    w = torch.exp(2.0 * torch.randn(B, H, cap, generator=g, **f32))
    s["score"] = torch.where(torch.rand(B, H, cap, generator=g, **f32) < 0.1, torch.zeros_like(w), w)
    # a cache that was evicted from before: each head holds positions of its own, in any order
    first = torch.argsort(torch.rand(B, H, cap, generator=g, **f32) +
                          (torch.arange(cap, device=DEV)[None, None, :] >= lens[:, None, None]), -1)
    s["slot_pos"] = (first * 3 // 2).to(torch.int32).contiguous()
    s["pos"] = lens * 3 // 2
    s["keep"] = torch.full((B,), case["keep"], **i32)
    s["score_out"] = torch.zeros(B, H, cap, **f32)
    s["pos_out"] = torch.zeros(B, H, cap, **i32)
    s["new_lens"] = torch.zeros(B, **i32)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _own_attend, "append": _own_append, "evict": _own_evict, "logprobs": _own_logprobs}[op](s)
    return {"attend": _attend, "append": _append, "evict": _evict, "logprobs": _logprobs}[op](s)


# -- the framework's calls -------------------------------------------------------


def _pages(s):
    """The cache's description, which a program makes once."""
    if "pages" not in s:
        from paper_2607_12422_amd import binding

        c = s["case"]
        s["pbd"] = binding
        s["pages"] = binding.make_pages(s["k"], s["v"], s["table"], n_q_heads=c["hq"], head_dim=c["hd"],
                                        score=s.get("score"), slot_pos=s.get("slot_pos"))
    return s["pbd"], s["pages"]


def _own_attend(s):
    pbd, pages = _pages(s)
    if "out" not in s:
        B, HQ, D = s["q"].shape
        s["max_len"] = s["table"].shape[1] * s["case"]["page"]
        s["out"] = torch.empty(B, HQ, D, dtype=torch.float32, device=DEV)
        s["lse"] = torch.empty(B, HQ, dtype=torch.float32, device=DEV)
        s["ws"] = torch.empty(pbd.pbd_paged_attention_workspace_bytes(pages, B, s["max_len"]), dtype=torch.uint8,
                              device=DEV)
    pbd.pbd_paged_attention(pages, s["q"], s["lens"], s["max_len"], s["out"], s["ws"], lse=s["lse"])
    r = dict(out=s["out"], lse=s["lse"])
    if s["score"] is not None:
        r["score"] = s["score"]
    return r


def _own_append(s):
    pbd, pages = _pages(s)
    pbd.pbd_paged_append(pages, s["new_k"], s["new_v"], s["lens"], s["pos"], s["rope"], q=s["q"], q_out=s["q_out"],
                         n_new=s["n_new"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, len_out=s["len_out"])
    return _append_outputs(s)


def _own_evict(s):
    pbd, pages = _pages(s)
    c = s["case"]
    if "ws" not in s:
        s["max_len"] = s["table"].shape[1] * c["page"]
        s["ws"] = torch.empty(pbd.pbd_paged_evict_workspace_bytes(pages, c["batch"], s["max_len"]),
                              dtype=torch.uint8, device=DEV)
    pbd.pbd_paged_evict(pages, s["lens"], s["max_len"], s["keep"], s["new_lens"], s["ws"], pos=s["pos"],
                        recent=c["recent"], sink=c["sink"], score_out=s["score_out"], slot_pos_out=s["pos_out"])
    return _evict_outputs(s)


def _own_logprobs(s):
    c = s["case"]
    if "pbd" not in s:
        from paper_2607_12422_amd import binding

        R, f32 = c["rows"], dict(dtype=torch.float32, device=DEV)
        s["pbd"] = binding
        s["logprob"], s["entropy"] = torch.empty(R, **f32), torch.empty(R, **f32)
        s["top_ids"] = torch.empty(R, c["top"], dtype=torch.int32, device=DEV) if c["top"] else None
        s["top_logprobs"] = torch.empty(R, c["top"], **f32) if c["top"] else None
        s["ws"] = torch.empty(binding.pbd_token_logprobs_workspace_bytes(R, c["vocab"], c["top"]),
                              dtype=torch.uint8, device=DEV)
    s["pbd"].pbd_token_logprobs(s["logits"], s["tokens"], s["logprob"], s["ws"], entropy=s["entropy"],
                                top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
    r = dict(logprob=s["logprob"], entropy=s["entropy"])
    if c["top"]:
        r.update(top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
    return r


# -- the plain forms -------------------------------------------------------------


def _blocks(s):
    """Both pools with their blocks opened: K [page][head][block][hd/E][16][E], V [...][hd/16][4][16][4]."""
    c = s["case"]
    e = 8 if c["dtype"] == "bf16" else 4
    n, D = c["page"] // 16, c["hd"]
    return (s["k"].unflatten(2, (n, D // e, 16, e)), s["v"].unflatten(2, (n, D // 16, 4, 16, 4)))


def _attend(s):
    c = s["case"]
    B, H, D = c["batch"], c["hkv"], c["hd"]
    k, v = _blocks(s)
    at = s["table"].clamp(min=0).long()
    k = k[at].permute(0, 2, 1, 3, 5, 4, 6).reshape(B, H, -1, D).float()
    v = v[at].permute(0, 2, 1, 3, 5, 7, 4, 6).reshape(B, H, -1, D).float()
    q = s["q"].reshape(B, H, -1, D)
    live = torch.arange(k.shape[2], device=DEV) < s["lens"][:, None, None, None]
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    x = torch.where(live, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    p = torch.where(l > 0, p / l, 0.0)
    r = dict(out=torch.matmul(p, v).reshape(B, -1, D), lse=(m + torch.log(l)).reshape(B, -1))
    if s["score"] is not None:
        s["score"] += p.sum(2)
        r["score"] = s["score"]
    return r


def _rotated(x, gain, rope):
    """Per-head RMSNorm (gain None: without) and rotate-half RoPE of [..., heads, hd]."""
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    a, b = x.chunk(2, -1)
    cos, sin = rope[..., None, :, 0], rope[..., None, :, 1]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _append(s):
    c = s["case"]
    B, R, H, D, page = c["batch"], c["rows"], c["hkv"], c["hd"], c["page"]
    k, v = _blocks(s)
    row = torch.arange(R, device=DEV)
    rope = s["rope"][s["pos"].long()[:, None] + row]
    new_k = _rotated(s["new_k"].unflatten(2, (H, D)), s["k_norm"], rope).to(s["k"].dtype)
    new_v = s["new_v"].unflatten(2, (H, D)).to(s["v"].dtype)
    q = _rotated(s["q"].unflatten(2, (-1, D)), s["q_norm"], rope).flatten(2)
    live = row < s["n_new"][:, None]
    s["q_out"].copy_(torch.where(live[:, :, None], q, s["q_out"]))
    b, r = live.nonzero(as_tuple=True)
    slot = s["lens"].long()[b] + r
    at, blk, i = s["table"].long()[b, slot // page], slot % page // 16, slot % 16
    k[at, :, blk, :, i] = new_k[b, r].unflatten(2, (k.shape[3], k.shape[5]))
    v[at, :, blk, :, i // 4, :, i % 4] = new_v[b, r].unflatten(2, (D // 16, 16))
    s["score"][b, :, slot] = 0.0
    s["slot_pos"][b, :, slot] = (s["pos"].long()[b] + r).to(torch.int32)[:, None]
    s["len_out"].copy_(s["lens"] + s["n_new"])
    return _append_outputs(s)


def _append_outputs(s):
    return dict(k=s["k"], v=s["v"], q=s["q_out"], score=s["score"], slot_pos=s["slot_pos"], lens=s["len_out"])


def _evict(s):
    c = s["case"]
    k, v = _blocks(s)
    page, n = c["page"], s["score"].shape[2]
    slot = torch.arange(n, device=DEV)
    lens, keep = s["lens"][:, None, None], torch.minimum(s["keep"], s["lens"])[:, None, None]
    stays = (s["slot_pos"] >= s["pos"][:, None, None] - c["recent"]) | (s["slot_pos"] < c["sink"])
    rank = torch.where(slot < lens, torch.where(stays, math.inf, s["score"]), -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(2, order, slot.expand_as(order))
    kept = place < keep
    # the i-th evicted slot below `keep` takes the i-th kept slot at or past it
    b, h, dst = (~kept & (slot < keep)).nonzero(as_tuple=True)
    _, _, src = (kept & (slot >= keep)).nonzero(as_tuple=True)
    to, td, ti = s["table"].long()[b, dst // page], dst % page // 16, dst % 16
    fr, fd, fi = s["table"].long()[b, src // page], src % page // 16, src % 16
    k[to, h, td, :, ti] = k[fr, h, fd, :, fi]
    v[to, h, td, :, ti // 4, :, ti % 4] = v[fr, h, fd, :, fi // 4, :, fi % 4]
    for name, out in (("score", "score_out"), ("slot_pos", "pos_out")):
        s[out].copy_(torch.where(slot < keep, s[name], s[out]))
        s[out][b, h, dst] = s[name][b, h, src]
    s["new_lens"].copy_(torch.minimum(s["keep"], s["lens"]))
    return _evict_outputs(s)


def _evict_outputs(s):
    return dict(k=s["k"], v=s["v"], score=s["score_out"], slot_pos=s["pos_out"], lens=s["new_lens"])


def _logprobs(s):
    top = s["case"]["top"]
    x = s["logits"].float()
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.double().sum(-1, keepdim=True)
    log_z = torch.log(z)
    chosen = d.gather(1, s["tokens"].long()[:, None]).double() - log_z
    mean = torch.where(e > 0, e * d, 0.0).double().sum(-1, keepdim=True) / z
    r = dict(logprob=chosen[:, 0].float(), entropy=(log_z - mean)[:, 0].float())
    if top:
        order = torch.sort(x, dim=-1, descending=True, stable=True)
        best, ids = order.values[:, :top], order.indices[:, :top]
        there = best > -math.inf
        r["top_ids"] = torch.where(there, ids, -1).to(torch.int32)
        r["top_logprobs"] = ((best - m).double() - log_z).float()
    return r


# -- what the calls cannot do without --------------------------------------------


def work(case):
    op, esz = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * esz + case["rows"] * (12 + 8 * case["top"]), "flops": 4 * n}
    B, H, HQ, D = case["batch"], case["hkv"], case["hq"], case["hd"]
    n = B * (case["lo"] + case["hi"]) / 2
    if op == "attend":
        b = n * H * D * 2 * esz + B * HQ * (2 * D + 1) * 4 + (8 * n * H if case["scored"] else 0)
        return {"bytes": b, "flops": 4 * n * HQ * D}
    if op == "append":
        rows = B * (max(1, case["rows"] // 2) + case["rows"]) / 2
        return {"bytes": rows * ((2 * HQ + 2 * H) * D * 4 + 2 * H * D * esz + 8 * H), "flops": rows * (HQ + H) * D * 6}
    mean = max(1.0, n / B)
    keep = min(case["keep"], mean)
    moved = B * H * keep * (1.0 - keep / mean)
    return {"bytes": n * H * 8 + B * H * keep * 8 + moved * 4 * D * esz, "flops": n * H}


# -- the same from the definitions, in 64 bits -----------------------------------


def _row_of(page, head, slot, case, value):
    """One slot's row of one head from a block's addresses, any of the arguments being index tensors."""
    D = case["hd"]
    e = 8 if case["dtype"] == "bf16" else 4
    d = torch.arange(D, device=DEV)
    slot = slot[..., None]
    block, i = slot % case["page"] // 16 * (16 * D), slot % 16
    where = (d // 16 * 256 + i // 4 * 64 + d % 16 * 4 + i % 4) if value else (d // e * 16 * e + i * e + d % e)
    return page[..., None], head, block + where


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        return _exact_logprobs(s)
    return {"attend": _exact_attend, "append": _exact_append, "evict": _exact_evict}[case["op"]](s)


def _exact_attend(s):
    c = s["case"]
    B, H, HQ, D = c["batch"], c["hkv"], c["hq"], c["hd"]
    out = torch.zeros(B, HQ, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, HQ), -math.inf, dtype=torch.float64, device=DEV)
    score = s["score"].double() if s["score"] is not None else None
    for b, n in enumerate(s["lens"].tolist()):
        slot = torch.arange(n, device=DEV)
        page = s["table"][b].long()[slot // c["page"]]
        for h in range(H):
            k = s["k"][_row_of(page, h, slot, c, False)].double()
            v = s["v"][_row_of(page, h, slot, c, True)].double()
            for g in range(h * (HQ // H), (h + 1) * (HQ // H)):
                if n:
                    x = (k * s["q"][b, g].double()).sum(-1) / math.sqrt(D)
                    lse[b, g] = torch.logsumexp(x, 0)
                    p = torch.exp(x - lse[b, g])
                    out[b, g] = (p[:, None] * v).sum(0)
                    if score is not None:
                        score[b, h, :n] += p
    r = dict(out=out, lse=lse)
    if score is not None:
        r["score"] = score
    return r


def _exact_append(s):
    c = s["case"]
    H, HQ, D, half = c["hkv"], c["hq"], c["hd"], c["hd"] // 2
    k, v, q = s["k"].double(), s["v"].double(), s["q_out"].double()
    score, slot_pos = s["score"].double(), s["slot_pos"].clone()

    def turned(x, gain, at):
        x = x.double().unflatten(-1, (-1, D))
        if gain is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * gain.double()
        t = torch.complex(x[..., :half], x[..., half:])
        t = t * torch.complex(at[:, :, 0], at[:, :, 1])[:, None]
        return torch.cat((t.real, t.imag), -1)

    for b, n in enumerate(s["n_new"].tolist()):
        first, pos = int(s["lens"][b]), int(s["pos"][b])
        at = s["rope"][pos : pos + n].double()
        slot = torch.arange(first, first + n, device=DEV)
        page = s["table"][b].long()[slot // c["page"]]
        new_k = turned(s["new_k"][b, :n], s["k_norm"], at)
        new_v = s["new_v"][b, :n].double().unflatten(-1, (H, D))
        q[b, :n] = turned(s["q"][b, :n], s["q_norm"], at).flatten(1)
        for h in range(H):
            k[_row_of(page, h, slot, c, False)] = new_k[:, h]
            v[_row_of(page, h, slot, c, True)] = new_v[:, h]
        score[b, :, first : first + n] = 0
        slot_pos[b, :, first : first + n] = torch.arange(pos, pos + n, device=DEV, dtype=torch.int32)
    return dict(k=k, v=v, q=q, score=score, slot_pos=slot_pos, lens=s["lens"] + s["n_new"])


def _exact_evict(s):
    c = s["case"]
    k, v = s["k"].double(), s["v"].double()
    score, pos = s["score_out"].double(), s["pos_out"].clone()
    for b, n in enumerate(s["lens"].tolist()):
        keep = min(c["keep"], n)
        table, last = s["table"][b].long(), int(s["pos"][b]) - c["recent"]
        w_all, p_all = s["score"][b, :, :n].double().cpu(), s["slot_pos"][b, :, :n].cpu()
        for h in range(c["hkv"]):
            p = p_all[h].numpy()
            w = w_all[h].clone().numpy()
            w[(p >= last) | (p < c["sink"])] = 1e300
            # ascending by (-weight, slot): the first `keep` stay
            by = (-w).argsort(kind="stable")[:keep]
            stays = set(by.tolist())
            dst = torch.tensor([i for i in range(keep) if i not in stays], dtype=torch.long, device=DEV)
            src = torch.tensor(sorted(i for i in stays if i >= keep), dtype=torch.long, device=DEV)
            score[b, h, :keep] = s["score"][b, h, :keep].double()
            pos[b, h, :keep] = s["slot_pos"][b, h, :keep]
            score[b, h, dst] = s["score"][b, h, src].double()
            pos[b, h, dst] = s["slot_pos"][b, h, src]
            to, fr = table[dst // c["page"]], table[src // c["page"]]
            for pool, value in ((k, False), (v, True)):
                pool[_row_of(to, h, dst, c, value)] = pool[_row_of(fr, h, src, c, value)]
    return dict(k=k, v=v, score=score, slot_pos=pos, lens=torch.minimum(s["keep"], s["lens"]))


def _exact_logprobs(s):
    top, V = s["case"]["top"], s["case"]["vocab"]
    logprob, entropy, ids, best = [], [], [], []
    for x, t in zip(s["logits"], s["tokens"].tolist()):
        x = x.double()
        y = x - torch.logsumexp(x, 0)
        logprob.append(y[t])
        entropy.append(-torch.special.xlogy(torch.exp(y), torch.exp(y)).sum())
        if top:
            # the highest logits, the lower id first among equal ones
            n = min(top, V)
            least = torch.topk(x, n).values[-1]
            some = (x >= least).nonzero()[:, 0]
            some = some[torch.sort(x[some], descending=True, stable=True).indices][:n]
            some = some[x[some] > -math.inf]
            fill = top - some.numel()
            ids.append(torch.nn.functional.pad(some, (0, fill), value=-1))
            best.append(torch.nn.functional.pad(y[some], (0, fill), value=-math.inf))
    r = dict(logprob=torch.stack(logprob), entropy=torch.stack(entropy))
    if top:
        r.update(top_ids=torch.stack(ids).to(torch.int32), top_logprobs=torch.stack(best))
    return r
