"""Refusals of the paged-cache and log-probability operators that need no GPU:
every argument the host can check is checked before anything is enqueued."""
import contextlib
import ctypes
import os

import pytest
import torch

import paged_ref as ref
from paper_2607_12422_amd import binding as b

P = 0x10000          # stands for a device pointer: never followed
INV, SHAPE, CAP = b.PBD_ERR_INVALID_ARG, b.PBD_ERR_SHAPE, b.PBD_ERR_CAPACITY


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2607_12422_amd import build
        build.build()
    return b.load_library()


def pages(**kw):
    d = dict(dtype=1, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=32, n_pages=9, page_stride=4096,
             head_stride=2048, k=P, v=P, table=P, table_width=4, score=P, slot_pos=P, slot_stride=128)
    d.update(kw)
    return b.PbdPages(**d)


BAD_PAGES = [
    (dict(dtype=2), INV), (dict(head_dim=96), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_q_heads=3), SHAPE),
    (dict(n_q_heads=512), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=8192), SHAPE),
    (dict(page_size=0), SHAPE), (dict(page_size=-32), SHAPE), (dict(n_pages=0), INV), (dict(page_stride=100), INV),
    (dict(head_stride=-1024), INV), (dict(k=0), INV), (dict(v=0), INV), (dict(table=0), INV), (dict(k=P + 2), INV),
    (dict(table_width=0), CAP), (dict(table_width=1 << 27), CAP), (dict(slot_stride=100), CAP), (dict(slot_stride=-1), CAP),
]


def attention(lib, pg, batch=2, q=P, q_stride=256, lens=P, max_len=128, scale=0.1, out=P, lse=None, ws=P, n=1 << 40):
    return lib.pbd_paged_attention(ctypes.byref(pg) if pg else None, batch, q, q_stride, lens, max_len, scale, out, lse,
                                   ws, n, None)


def append(lib, pg, batch=2, max_new=3, q=P, k=P, v=P, stride=512, lens=P, n_new=P, pos=P, qn=P, kn=P, eps=1e-6, rope=P,
           rope_len=100, q_out=P, lens_out=P + 64):
    return lib.pbd_paged_append(ctypes.byref(pg) if pg else None, batch, max_new, q, k, v, stride, lens, n_new, pos, qn,
                                kn, eps, rope, rope_len, q_out, lens_out, None)


def evict(lib, pg, batch=2, lens=P, max_len=128, keep=P, pos=P, recent=1, sink=1, so=P, po=P, new=P, ws=P, n=1 << 40):
    return lib.pbd_paged_evict(ctypes.byref(pg) if pg else None, batch, lens, max_len, keep, pos, recent, sink, so, po,
                               new, ws, n, None)


def logprobs(lib, rows=3, vocab=100, dtype=0, x=P, stride=100, tok=P, n=2, lp=P, ent=P, ids=P, best=P, ws=P, size=1 << 40):
    return lib.pbd_token_logprobs(rows, vocab, dtype, x, stride, tok, n, lp, ent, ids, best, None, ws, size, None)


@pytest.mark.parametrize("call", [attention, append, evict])
def test_descriptions_of_the_cache(lib, call):
    assert call(lib, None) == INV
    for kw, code in BAD_PAGES:
        if call is append and kw == dict(slot_stride=100):
            continue                       # no bound on the lengths: the device checks them
        assert call(lib, pages(**kw)) == code, kw
        assert b.pbd_last_error()
    for batch, code in ((0, INV), (-1, INV), (65536, CAP)):
        assert call(lib, pages(), batch=batch) == code


def test_attention(lib):
    for kw, code in [(dict(q=0), INV), (dict(lens=0), INV), (dict(out=0), INV), (dict(ws=0), INV), (dict(q=P + 4), INV),
                     (dict(out=P + 8), INV), (dict(ws=P + 8), INV), (dict(q_stride=252), INV), (dict(q_stride=257), INV),
                     (dict(max_len=0), INV), (dict(max_len=129), CAP), (dict(scale=0.0), INV),
                     (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(n=100), CAP)]:
        assert attention(lib, pages(), **kw) == code, kw
    assert b.pbd_paged_attention_workspace_bytes(pages(), 2, 0) == 0
    assert b.pbd_paged_attention_workspace_bytes(pages(), 2, 129) == 0
    plain = b.pbd_paged_attention_workspace_bytes(pages(score=0, slot_pos=0), 2, 128)
    assert 0 < plain < b.pbd_paged_attention_workspace_bytes(pages(), 2, 128)


def test_append(lib):
    for kw in [dict(k=0), dict(v=0), dict(lens=0), dict(pos=0), dict(rope=0), dict(q=0), dict(q_out=0),
               dict(q=0, q_out=0), dict(max_new=-1), dict(max_new=1 << 21), dict(rope_len=0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(stride=255), dict(stride=258), dict(stride=252),
               dict(q=P + 4), dict(k=P + 4), dict(v=P + 8), dict(rope=P + 8), dict(q_out=P + 4), dict(qn=P + 2),
               dict(kn=P + 2), dict(lens_out=P)]:
        assert append(lib, pages(), **kw) == INV, kw


def test_evict(lib):
    for kw, code in [(dict(lens=0), INV), (dict(keep=0), INV), (dict(so=0), INV), (dict(new=0), INV), (dict(ws=0), INV),
                     (dict(po=0), INV), (dict(pos=0), INV), (dict(recent=-1), INV), (dict(sink=-1), INV),
                     (dict(max_len=0), INV), (dict(max_len=129), CAP), (dict(ws=P + 4), INV), (dict(n=16), CAP)]:
        assert evict(lib, pages(), **kw) == code, kw
    assert evict(lib, pages(score=0)) == INV
    assert evict(lib, pages(slot_pos=0)) == INV
    assert evict(lib, pages(slot_pos=0), recent=0, sink=0, pos=0) == INV          # slot_pos_out without slot_pos


def test_logprobs(lib):
    for kw, code in [(dict(rows=0), INV), (dict(rows=(1 << 22) + 1), INV), (dict(vocab=0), INV),
                     (dict(vocab=(1 << 22) + 1), INV), (dict(n=-1), INV), (dict(n=33), INV), (dict(dtype=3), INV),
                     (dict(x=0), INV), (dict(ws=0), INV), (dict(tok=0), INV), (dict(lp=0), INV), (dict(ids=0), INV),
                     (dict(best=0), INV), (dict(stride=99), INV), (dict(x=P + 2), INV), (dict(dtype=1, x=P + 1), INV),
                     (dict(ws=P + 8), INV), (dict(size=0), CAP)]:
        assert logprobs(lib, **kw) == code, kw
    assert b.pbd_token_logprobs_workspace_bytes(0, 10, 1) == 0
    assert b.pbd_token_logprobs_workspace_bytes(1, 10, 33) == 0


def test_calls_reject_null_context(lib):
    pg = pages()
    assert lib.pbd_context_pages(None, ctypes.byref(pg)) == INV
    assert lib.pbd_decode_paged(None, ctypes.byref(pg), 1, P, P, P, 1, 0, None, P, 1 << 30, None) == INV
    assert lib.pbd_decode_paged_workspace_bytes(None, ctypes.byref(pg), 1, 1) == 0


def test_struct_layout_matches_header():
    assert ctypes.sizeof(b.PbdPages) == 120
    assert (b.PbdPages.page_stride.offset, b.PbdPages.k.offset, b.PbdPages.table_width.offset,
            b.PbdPages.score.offset, b.PbdPages.status.offset) == (24, 48, 72, 80, 112)


@contextlib.contextmanager
def refused():
    """A refusal for the argument's sake (host tensors alone are one, too)."""
    with pytest.raises(b.PbdError) as e:
        yield
    assert "must be on a GPU" not in str(e.value)


def test_binding_checks_shapes_and_types():
    """make_pages and the calls refuse tensors that do not hold what the library would read."""
    c = ref.Cache([40, 10], 2, 64, torch.bfloat16)
    ok = dict(n_q_heads=4, head_dim=64)
    pg = b.make_pages(c.k, c.v, c.table, **ok)
    assert (pg.page_size, pg.n_pages, pg.page_stride, pg.head_stride) == (16, c.k.shape[0], 2 * 1024, 1024)
    score, pos = torch.zeros(2, 2, 48), torch.zeros(2, 2, 48, dtype=torch.int32)
    assert b.make_pages(c.k, c.v, c.table, score=score, slot_pos=pos, **ok).slot_stride == 48
    for args, kw in [((c.k, c.v[:5], c.table), {}), ((c.k, c.v.float(), c.table), {}), ((c.k, c.v, c.table.long()), {}),
                     ((c.k, c.v, c.table[:, ::2]), {}), ((c.k.half(), c.v.half(), c.table), {}),
                     ((c.k, c.v, c.table), dict(score=score.double())), ((c.k, c.v, c.table), dict(score=score[:1])),
                     ((c.k, c.v, c.table), dict(slot_pos=pos, score=score[..., :9])), ((c.k[:, :, :40], c.v[:, :, :40], c.table), {}),
                     ((c.k, c.v, c.table), dict(status=torch.zeros(2, dtype=torch.int32)))]:
        with refused():
            b.make_pages(*args, **ok, **kw)
    lens, q, out = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, 64), torch.zeros(2, 4, 64)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for a in [(q[:1], lens, out, ws), (q.double(), lens, out, ws), (q, lens.long(), out, ws), (q, lens, out[:1], ws),
              (q.transpose(1, 2).contiguous().transpose(1, 2), lens, out, ws), (q, lens, out.bfloat16(), ws),
              (torch.zeros(3, 4, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 4, 64), ws)]:
        with refused():
            b.pbd_paged_attention(pg, a[0], a[1], 48, a[2], a[3])
    k, rope = torch.zeros(2, 3, 128), torch.zeros(9, 32, 2)
    for a, kw in [((k, k[:, :2], lens, lens, rope), {}), ((k, k, lens, lens, rope[:, :16]), {}),
                  ((k, k.double(), lens, lens, rope), {}), ((k, k, lens[:1], lens, rope), {}),
                  ((k, k, lens, lens, rope), dict(q=torch.zeros(2, 3, 128), q_out=torch.zeros(2, 3, 256))),
                  ((k, torch.zeros(2, 3, 256)[..., :128], lens, lens, rope), {}),
                  ((k, k, lens, lens, rope), dict(k_norm=torch.zeros(64)))]:
        with refused():
            b.pbd_paged_append(pg, *a, **kw)
    x, t, lp = torch.zeros(4, 100), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for a, kw in [((x.half(), t, lp, ws), {}), ((x, t.long(), lp, ws), {}), ((x, t, lp[:2], ws), {}),
                  ((x.t(), torch.zeros(100, dtype=torch.int32), torch.zeros(100), ws), {}),
                  ((x, t, lp, ws), dict(top_ids=torch.zeros(4, 3, dtype=torch.int32), top_logprobs=torch.zeros(4, 2)))]:
        with refused():
            b.pbd_token_logprobs(*a, **kw)


def test_host_tensors_and_layers_out_of_range():
    c = ref.Cache([40, 10], 2, 64, torch.bfloat16)
    pg = b.make_pages(c.k, c.v, c.table, n_q_heads=4, head_dim=64, score=torch.zeros(2, 2, 48))
    lens, ws = torch.zeros(2, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    k, rope = torch.zeros(2, 3, 128), torch.zeros(9, 32, 2)
    for call in (lambda: b.pbd_paged_attention(pg, torch.zeros(2, 4, 64), lens, 48, torch.zeros(2, 4, 64), ws),
                 lambda: b.pbd_paged_append(pg, k, k, lens, lens, rope),
                 lambda: b.pbd_paged_evict(pg, lens, 48, lens, lens.clone(), ws),
                 lambda: b.pbd_token_logprobs(torch.zeros(2, 100), lens, torch.zeros(2), ws)):
        with pytest.raises(b.PbdError, match="must be on a GPU"):
            call()
    with refused():
        b.layer_pages(pg, 0)
    k, v = (torch.stack((t, t)) for t in (c.k, c.v))
    both = b.make_pages(k, v, c.table, n_q_heads=4, head_dim=64)
    assert b.layer_pages(both, 1).k == k[1].data_ptr() and b.layer_pages(both, 1).v == v[1].data_ptr()
    for layer in (-1, 2):
        with refused():
            b.layer_pages(both, layer)


def test_launches_past_the_largest_grid(lib):
    """Sizes within the other limits whose launches would have 2^32 threads or more: refused before anything runs."""
    far = dict(page_size=4096, table_width=1 << 18, slot_stride=1 << 30, page_stride=4096 * 64 * 16, head_stride=4096 * 64)
    big = dict(far, n_kv_heads=16, n_q_heads=16)
    n = 1 << 30
    assert attention(lib, pages(**big), batch=1, q_stride=1024, max_len=n) == CAP
    assert b.pbd_last_error()
    assert b.pbd_paged_attention_workspace_bytes(pages(**big), 1, n) == 0
    assert b.pbd_paged_attention_workspace_bytes(pages(**big), 1, n - 2048) > 0
    assert b.pbd_paged_attention_workspace_bytes(pages(**dict(big, score=0)), 1, n) > 0
    assert evict(lib, pages(**far), batch=1, max_len=n) == CAP
    assert b.pbd_paged_evict_workspace_bytes(pages(**far), 1, n) == 0
    assert b.pbd_paged_evict_workspace_bytes(pages(**far), 1, n - 4096) > 0
    assert logprobs(lib, rows=1 << 22, vocab=1 << 20, stride=1 << 20) == CAP
    assert b.pbd_token_logprobs_workspace_bytes(1 << 22, 1 << 20, 1) == 0
    assert b.pbd_token_logprobs_workspace_bytes(1 << 22, 152000, 1) > 0


def test_decoding_over_a_cache_on_another_device():
    """The context's buffers lie on its own device: a cache on another one is refused."""
    class On:
        """Stands for an int32 tensor on a device."""
        dtype, nbytes = torch.int32, 1 << 20

        def __init__(self, device):
            self.device = device

        def numel(self):
            return 2

        def get_device(self):
            return self.device

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return P

    class Tiny:
        n_layers, vocab = 1, 100

    c = ref.Cache([40, 10], 2, 64, torch.bfloat16)
    pg = b.make_pages(c.k, c.v, c.table, n_q_heads=4, head_dim=64)
    pg.device = 1
    eng = object.__new__(b.Engine)
    eng.lib, eng.ctx, eng.cfg, eng.kv = b.load_library(), None, Tiny, On(0)
    t = [On(1) for _ in range(3)]
    with pytest.raises(b.PbdError, match="context's device"):
        eng.pbd_decode_paged(pg, *t, 48, On(1))
