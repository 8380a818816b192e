"""pbd_decode_paged and the operators around it as a serving loop uses them:
prefill, paged decoding, eviction in every layer, decoding on, log
probabilities of what was decoded.  Each token is checked against a plain
64-bit decoder that reads the cache the GPU had; logits within the bounds that
the other passes are held to (tiny fp32 1e-4, bf16 2e-2)."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
import synth
from gpu_harness import GpuRun, decisive
from oracle import model as om
from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TINY = synth.TINY
BF16 = synth.QWEN3_0_6B.with_(n_layers=2, vocab=4096)


def plain_token(m, tok, pos, cache, adapter=False):
    """One token at position pos over cache[l] = (K, V) [n][n_kv][d] (keys rotated): (logits, new K/V per layer,
    weights [l][n_kv][n + 1] summed over the query heads of each KV head)."""
    cfg = m.cfg
    d, G = cfg.head_dim, cfg.n_q_heads // cfg.n_kv_heads
    x = m.embed[[tok]]
    new, weights = [], []
    for lw, (ck, cv) in zip(m.layers, cache):
        xn = om.rms_norm(x, lw["attn_norm"], cfg.rms_eps)
        q, k, v = (m.linear(lw, n, xn, adapter).reshape(1, -1, d) for n in ("q", "k", "v"))
        if cfg.qk_norm:
            q, k = om.rms_norm(q, lw["q_norm"], cfg.rms_eps), om.rms_norm(k, lw["k_norm"], cfg.rms_eps)
        q, k = om.rope(q, np.array([pos]), cfg.rope_theta), om.rope(k, np.array([pos]), cfg.rope_theta)
        K, V = np.concatenate([ck, k]), np.concatenate([cv, v])
        p = np.stack([om.softmax_rows((K[:, h // G] @ q[0, h]) / np.sqrt(d)) for h in range(cfg.n_q_heads)])
        o = np.stack([p[h] @ V[:, h // G] for h in range(cfg.n_q_heads)])
        x = x + m.linear(lw, "o", o.reshape(1, -1), adapter)
        xm = om.rms_norm(x, lw["mlp_norm"], cfg.rms_eps)
        x = x + m.linear(lw, "down", om.silu(m.linear(lw, "gate", xm, adapter)) * m.linear(lw, "up", xm, adapter), adapter)
        new.append((k[0], v[0]))
        weights.append(p.reshape(cfg.n_kv_heads, G, -1).sum(1))
    return m.logits(x)[0], new, weights


class Server:
    """An engine after its prefill and a paged cache: the context's own, or a pool with pages of another size."""

    def __init__(self, cfg, lengths, extra=64, own_pool=0, seed=50, max_batch=None, scored=True):
        self.cfg, self.tol = cfg, 1e-4 if cfg.dtype == "f32" else 2e-2
        w = synth.make_weights(cfg, seed)
        self.m = om.OracleModel(w)
        self.B = len(lengths)
        max_seq = max(lengths) + cfg.width + extra
        self.g = GpuRun(cfg, w, max_batch=max_batch or self.B, max_seq=max_seq,
                        prefill_chunk=min(64, 4096 // (max_batch or self.B)))
        self.g.prefill(synth.make_prompts(cfg, lengths, seed + 1))
        self.eng = self.g.eng
        self.L, self.H, self.D = cfg.n_layers, cfg.n_kv_heads, cfg.head_dim
        self.dtype = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
        nblk = -(-max_seq // 16)
        Bm = max_batch or self.B
        self.dense = self.eng.kv.view(self.dtype).view(2, self.L, Bm, self.H, nblk, 16 * self.D)
        cap = nblk * 16
        self.score = torch.zeros(self.L, self.B, self.H, cap, device=DEV) if scored else None
        self.slot_pos = torch.arange(cap, dtype=torch.int32, device=DEV).expand(self.L, self.B, self.H, cap).contiguous() \
            if scored else None
        if own_pool:
            # pages of own_pool positions anywhere in a pool, the prefix's blocks copied in
            per = own_pool // 16
            width = -(-nblk // per)
            n = self.B * width + 5
            self.table = torch.randperm(n, generator=torch.Generator().manual_seed(1))[: self.B * width]
            self.table = self.table.to(torch.int32).view(self.B, width).to(DEV)
            self.pool = torch.full((2, self.L, n, self.H, own_pool * self.D), math.nan, dtype=self.dtype, device=DEV)
            for b in range(self.B):
                for i in range(-(-lengths[b] // 16)):
                    at = (i % per) * 16 * self.D
                    self.pool[:, :, int(self.table[b, i // per]), :, at: at + 16 * self.D] = self.dense[:, :, b, :, i]
            self.page = own_pool
            self.cap = min(cap, width * own_pool)
            self.pages = pbd.make_pages(self.pool[0], self.pool[1], self.table, n_q_heads=cfg.n_q_heads,
                                        head_dim=self.D, score=self.score, slot_pos=self.slot_pos)
        else:
            self.pool, self.page, self.cap = None, 16, cap
            # the sequences' rows of the default table
            table = self.eng.pbd_context_pages().keep[1][: self.B].contiguous()
            self.pages = self.eng.pbd_context_pages(table, score=self.score, slot_pos=self.slot_pos)
        self.token, self.pos = self.g.anchor.clone(), self.g.seq_len.clone()
        self.len = self.g.seq_len.clone()
        self.logits = torch.zeros(self.B, cfg.vocab, device=DEV)
        self.ws = torch.full((self.eng.pbd_decode_paged_workspace_bytes(self.pages, self.B, self.cap),), 0xFF,
                             dtype=torch.uint8, device=DEV)
        mk, mv = ref.block_maps(self.D, 8 if cfg.dtype == "bf16" else 4)
        self.maps = mk, mv

    def cache(self, b, n):
        """[l] -> (K, V) [n][H][D] float64 of sequence b's first n slots."""
        slot = torch.arange(n)
        ik, iv = self.maps[0][slot % 16], self.maps[1][slot % 16]
        out = []
        for l in range(self.L):
            kv = []
            for which, i in ((0, ik), (1, iv)):
                if self.pool is None:
                    src = self.dense[which, l, b].cpu()                       # [H][nblk][16 D]
                    x = src[:, slot // 16]
                else:
                    pg = self.table[b].cpu().long()[slot // self.page]
                    x = self.pool[which, l].cpu()[pg].unflatten(2, (-1, 16 * self.D))
                    x = x[torch.arange(n), :, slot % self.page // 16].transpose(0, 1)
                kv.append(torch.gather(x, 2, i[None].expand(self.H, -1, -1)).transpose(0, 1).double().numpy())
            out.append(tuple(kv))
        return out

    def call(self, flags=0):
        self.eng.pbd_decode_paged(self.pages, self.token, self.pos, self.len, self.cap, self.ws, logits=self.logits,
                                  flags=flags)

    def step(self, flags=0, run=None):
        """One decode call, checked."""
        tok, pos, n = (t.cpu().tolist() for t in (self.token, self.pos, self.len))
        caches = [self.cache(b, n[b]) for b in range(self.B)]
        score = None if self.score is None else self.score.cpu().double().numpy()
        (run or self.call)(*(() if run else (flags,)))
        torch.cuda.synchronize()
        lg = self.logits.cpu().double().numpy()
        worst = 0.0
        for b in range(self.B):
            want, new, weights = plain_token(self.m, tok[b], pos[b], caches[b], bool(flags & pbd.PBD_PASS_ADAPTER_ON))
            worst = max(worst, float(np.abs(lg[b] - want).max()))
            assert worst <= self.tol, (b, worst)
            if decisive(want[None], self.tol)[0]:
                assert int(self.token[b]) == int(np.argmax(want))
            assert int(self.token[b]) == int(lg[b].argmax())
            assert int(self.pos[b]) == pos[b] + 1 and int(self.len[b]) == n[b] + 1
            now = self.cache(b, n[b] + 1)
            for l in range(self.L):
                for i in range(2):
                    assert np.array_equal(now[l][i][:-1], caches[b][l][i])
                    assert np.abs(now[l][i][-1] - new[l][i]).max() <= self.tol * max(1, np.abs(new[l][i]).max())
                if score is not None:
                    got = self.score[l, b].cpu().double().numpy()
                    s0 = score[l, b].copy()
                    s0[:, n[b]] = 0
                    s0[:, : n[b] + 1] += weights[l]
                    assert np.abs(got - s0).max() <= self.tol
                    assert torch.all(self.slot_pos[l, b, :, n[b]] == pos[b])
        assert self.g.status() == 0
        return tok


@pytest.mark.parametrize("own_pool", [0, 64])
@pytest.mark.parametrize("cfg,lengths", [(TINY, [40]), (TINY, [5, 70, 33]), (BF16, [130]), (BF16, [20, 100, 64])])
def test_tokens(cfg, lengths, own_pool):
    s = Server(cfg, lengths, own_pool=own_pool)
    for i in range(4):
        s.step(flags=pbd.PBD_PASS_ADAPTER_ON if i == 2 else 0)
    s.g.close()


@pytest.mark.parametrize("cfg", [TINY.with_(block=0), BF16.with_(block=0)])
def test_as_the_dense_single_token_step(cfg):
    """The same tokens' logits as pbd_verify_block at D = 0, within the passes' bound; then the dense passes go on
    over the cache that the paged ones left."""
    lengths = [50, 21]
    a = Server(cfg, lengths, scored=False)
    b = Server(cfg, lengths, scored=False)
    for i in range(6):
        seq, tok = a.pos.clone(), a.token.clone()
        a.call()
        v, lg = torch.zeros(2, 1, dtype=torch.int32, device=DEV), torch.zeros(2, 1, cfg.vocab, device=DEV)
        eng = a.eng if i == 5 else b.eng          # at the end: the dense step on the paged cache's context
        if i == 5:
            again = torch.zeros(2, 1, cfg.vocab, device=DEV)
            b.eng.pbd_verify_block(seq, tok, torch.zeros(2, 1, dtype=torch.int32, device=DEV), v, again)
        eng.pbd_verify_block(seq, tok, torch.zeros(2, 1, dtype=torch.int32, device=DEV), v, lg)
        torch.cuda.synchronize()
        assert float((a.logits - lg[:, 0]).abs().max()) <= a.tol
        if i == 5:
            assert float((again - lg).abs().max()) <= a.tol
    for s in (a, b):
        assert s.g.status() == 0
        s.g.close()


def test_large_batch():
    """Passes of 128 rows and more take fp16 operands; the sequences are a subset of the context's slots."""
    lengths = [3 + 5 * i % 40 for i in range(130)]
    s = Server(BF16.with_(block=2), lengths, extra=30, max_batch=133)
    s.step()
    s.g.close()


@pytest.mark.parametrize("cfg,own_pool", [(TINY, 0), (TINY, 32), (BF16, 64)])
def test_serving_loop(cfg, own_pool):
    """Decode, evict every layer to a budget, decode on by a captured graph, log probabilities of each token."""
    s = Server(cfg, [90, 40, 130], own_pool=own_pool)
    for _ in range(3):
        s.step()
    keep = torch.full((3,), 64, dtype=torch.int32, device=DEV)
    ews = torch.empty(pbd.pbd_paged_evict_workspace_bytes(s.pages, 3, s.cap), dtype=torch.uint8, device=DEV)
    before = s.len.tolist()
    new = torch.zeros(3, dtype=torch.int32, device=DEV)
    held = []
    for l in range(s.L):
        held.append([(s.score[l, b].cpu(), s.slot_pos[l, b].cpu()) for b in range(3)])
        pbd.pbd_paged_evict(pbd.layer_pages(s.pages, l), s.len, s.cap, keep, new, ews, pos=s.pos, recent=8, sink=2)
    s.len.copy_(new)
    torch.cuda.synchronize()
    assert new.tolist() == [64, 43, 64]
    for l in range(s.L):
        for b, n in enumerate(before):
            score, pos = held[l][b]
            for h in range(s.H):
                stay, _ = ref.kept(score[h].tolist(), pos[h].tolist(), n, 64, int(s.pos[b]) - 8, 2)
                got = sorted(s.slot_pos[l, b, h, : len(stay)].tolist())
                assert got == sorted(pos[h][stay].tolist())
    s.step()
    graph = torch.cuda.CUDAGraph()
    state = [t.clone() for t in (s.token, s.pos, s.len)]
    with torch.cuda.graph(graph):
        s.call()
    for t, t0 in zip((s.token, s.pos, s.len), state):
        assert torch.equal(t, t0)
    lp, H = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV)
    ids, best = torch.zeros(3, 5, dtype=torch.int32, device=DEV), torch.zeros(3, 5, device=DEV)
    lws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(3, cfg.vocab, 5), dtype=torch.uint8, device=DEV)
    for _ in range(4):
        s.step(run=graph.replay)
        pbd.pbd_token_logprobs(s.logits, s.token, lp, lws, entropy=H, top_ids=ids, top_logprobs=best)
        y = torch.log_softmax(s.logits.double(), -1)
        assert torch.equal(ids[:, 0], s.token) and torch.equal(lp, best[:, 0])
        assert float((lp - y.gather(1, s.token.long()[:, None])[:, 0]).abs().max()) <= 1e-5
        assert float((H + (y.exp() * y).sum(-1)).abs().max()) <= 1e-4
    s.g.close()


def test_committed_tokens_of_a_speculative_step():
    """Log probabilities of what a verify pass committed: its logits against pbd_accept_commit's out_tokens, whose
    entries past the accepted ones (-1) are skipped."""
    cfg = TINY
    g = GpuRun(cfg, synth.make_weights(cfg, 70), max_batch=2, max_seq=200)
    g.prefill(synth.make_prompts(cfg, [60, 31], 71))
    d, _ = g.draft()
    v, lg = g.verify(d)
    n, out = g.accept(d, v, forced=[3, 0])
    W = cfg.width
    lp = torch.full((2, W), 77.0, device=DEV)
    ws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(2 * W, cfg.vocab, 0), dtype=torch.uint8, device=DEV)
    pbd.pbd_token_logprobs(lg, out, lp, ws)
    y = torch.log_softmax(lg.double(), -1)
    for b, k in enumerate((3, 0)):
        want = y[b, : k + 1].gather(1, out[b, : k + 1].long()[:, None])[:, 0]
        assert float((lp[b, : k + 1] - want).abs().max()) <= 1e-5
        assert torch.all(lp[b, k + 1:] == 77.0)
    g.close()


def test_invalid_sequences_are_skipped():
    s = Server(TINY, [40, 30, 20, 50, 25], scored=False)
    tok, pos, n = s.token.clone(), s.pos.clone(), s.len.clone()
    kv = s.eng.kv.clone()
    s.token[1] = TINY.vocab
    s.pos[2] = s.g.eng.pcfg.max_seq
    s.len[3] = s.cap
    table = s.pages.keep[1].clone()
    table[4, 1] = -5
    s.pages = s.eng.pbd_context_pages(table)
    tok, pos, n = s.token.clone(), s.pos.clone(), s.len.clone()
    s.call()
    torch.cuda.synchronize()
    assert s.g.status() == pbd.PBD_STATUS_TOKEN | pbd.PBD_STATUS_CAPACITY | pbd.PBD_STATUS_PAGE
    assert (s.pos - pos).tolist() == [1, 0, 0, 0, 0] and (s.len - n).tolist() == [1, 0, 0, 0, 0]
    assert torch.equal(s.token[1:], tok[1:])
    was = kv.view(s.dtype).view_as(s.dense)
    assert torch.equal(s.dense[:, :, 1:], was[:, :, 1:]) and not torch.equal(s.dense[:, :, 0], was[:, :, 0])
    s.g.close()


def test_refusals_on_a_live_context():
    """What the host can see is refused before anything runs: tokens, lengths, caches and the status stay."""
    import ctypes
    s = Server(TINY, [40, 30], own_pool=32)
    lib, ctx = s.eng.lib, s.eng.ctx
    INV, SHAPE, CAP = pbd.PBD_ERR_INVALID_ARG, pbd.PBD_ERR_SHAPE, pbd.PBD_ERR_CAPACITY
    n, most = s.ws.numel(), s.pages.table_width * s.page
    before = [t.clone() for t in (s.token, s.pos, s.len, s.pool, s.eng.kv, s.score, s.slot_pos, s.logits)]

    def call(batch=2, token=s.token.data_ptr(), pos=s.pos.data_ptr(), length=s.len.data_ptr(), max_len=s.cap, flags=0,
             logits=s.logits.data_ptr(), ws=s.ws.data_ptr(), size=n, **kw):
        p = pbd.PbdPages.from_buffer_copy(s.pages)
        for k, x in kw.items():
            setattr(p, k, x)
        return lib.pbd_decode_paged(ctx, ctypes.byref(p), batch, token, pos, length, max_len, flags, logits, ws, size, None)

    other = s.pages.state_layer_stride
    for kw, code in [(dict(batch=0), INV), (dict(batch=3), CAP), (dict(token=None), INV), (dict(pos=None), INV),
                     (dict(length=None), INV), (dict(ws=None), INV), (dict(token=s.pos.data_ptr()), INV),
                     (dict(length=s.pos.data_ptr()), INV), (dict(length=s.token.data_ptr()), INV), (dict(max_len=0), INV),
                     (dict(max_len=most + 1), CAP), (dict(max_len=-1), CAP), (dict(ws=s.ws.data_ptr() + 8), INV),
                     (dict(size=n - 1), CAP), (dict(flags=pbd.PBD_PASS_MASK_BLOCK), INV),
                     (dict(flags=pbd.PBD_PASS_MASK_CAUSAL), INV),
                     (dict(flags=pbd.PBD_PASS_ADAPTER_ON | pbd.PBD_PASS_ADAPTER_OFF), INV), (dict(flags=1 << 30), INV),
                     (dict(dtype=pbd.PBD_DTYPE_BF16), SHAPE), (dict(n_q_heads=2 * TINY.n_q_heads), SHAPE),
                     (dict(n_kv_heads=1, n_q_heads=TINY.n_q_heads), SHAPE), (dict(head_dim=128), SHAPE),
                     (dict(layer_stride=0), INV), (dict(layer_stride=-1024), INV), (dict(layer_stride=1000), INV),
                     (dict(state_layer_stride=0), INV), (dict(state_layer_stride=-other), INV),
                     (dict(k=None), INV), (dict(table=None), INV), (dict(page_size=24), SHAPE), (dict(n_pages=0), INV),
                     (dict(slot_stride=s.cap - 1), CAP)]:
        assert call(**kw) == code, kw
        assert pbd.pbd_last_error(ctx)
    # the binding's own: a table of fewer sequences, another number of layers, types
    for args, kw in [((torch.cat((s.token, s.token)), s.pos, s.len), {}), ((s.token, s.pos.long(), s.len), {}),
                     ((s.token, s.pos, s.len[:1]), {}), ((s.token, s.pos, s.len), dict(logits=s.logits[:1])),
                     ((s.token, s.pos, s.len), dict(logits=s.logits.double()))]:
        with pytest.raises(pbd.PbdError):
            s.eng.pbd_decode_paged(s.pages, *args, s.cap, s.ws, **kw)
    few = pbd.make_pages(s.pool[0][:1], s.pool[1][:1], s.table, n_q_heads=TINY.n_q_heads, head_dim=s.D)
    with pytest.raises(pbd.PbdError):
        s.eng.pbd_decode_paged(few, s.token, s.pos, s.len, s.cap, s.ws)
    torch.cuda.synchronize()
    bits = lambda t: t.contiguous().view(torch.uint8)
    for t, t0 in zip((s.token, s.pos, s.len, s.pool, s.eng.kv, s.score, s.slot_pos, s.logits), before):
        assert torch.equal(bits(t), bits(t0))
    assert s.g.status() == 0
    s.step()
    s.g.close()
