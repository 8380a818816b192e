"""Refusals of the packed-row operators that need no GPU: every argument the host can check is checked before anything is
enqueued; and the plain allocator that the GPU tests compare with."""
import ctypes
import os

import pytest
import torch

import rows_ref as rr
from paper_2607_12422_amd import binding as b
from test_paged_abi import BAD_PAGES, CAP, INV, P, SHAPE, pages

UNS = b.PBD_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2607_12422_amd import build
        build.build()
    return b.load_library()


def plain(**kw):
    return pages(**dict(dict(score=0, slot_pos=0), **kw))


def ref(pg):
    return ctypes.byref(pg) if pg else None


def plan(lib, batch=2, page=32, n_pages=9, table=P, width=4, seq=P + 64, free=P, n_free=P, lens=P, new=P + 256, pos=P, rows=10,
         start=P + 512, row_seq=P, row_pos=P, slots=P, new_lens=P + 1024, status=None):
    return lib.pbd_page_plan(batch, page, n_pages, table, width, seq, free, n_free, lens, new, pos, rows, start, row_seq, row_pos,
                             slots, new_lens, status, None)


def release(lib, batch=2, page=32, n_pages=9, table=P, width=4, seq=P, free=P, n_free=P, keep=P + 64, status=None):
    return lib.pbd_page_release(batch, page, n_pages, table, width, seq, free, n_free, keep, status, None)


def append(lib, pg, rows=3, q=P, k=P, v=P, stride=512, slots=P, pos=P, qn=P, kn=P, eps=1e-6, rope=P, rope_len=100, q_out=P,
           batch=None):
    return lib.pbd_paged_append_rows(ref(pg), rows, q, k, v, stride, slots, pos, qn, kn, eps, rope, rope_len, q_out, None)


def packed(lib, pg, batch=2, rows=5, q=P, stride=256, start=P, lens=P, max_len=128, scale=0.1, out=P + (1 << 20), lse=None, ws=P, n=1 << 40):
    return lib.pbd_packed_attention(ref(pg), batch, rows, q, stride, start, lens, max_len, scale, out, lse, ws, n, None)


def tree(lib, pg, batch=2, rows=5, q=P, stride=256, start=P, lens=P, mask=P, max_len=128, scale=0.1, out=P + (1 << 20), lse=None, ws=P,
         n=1 << 40):
    return lib.pbd_tree_attention(ref(pg), batch, rows, q, stride, start, lens, mask, max_len, scale, out, lse, ws, n, None)


def layout(lib, batch=2, rows=5, start=P, parent=P, pos=P, mask=P, row_pos=P):
    return lib.pbd_tree_layout(batch, rows, start, parent, pos, mask, row_pos, None, None)


def commit(lib, pg, layers=1, batch=2, rows=5, start=P, lens=P, parent=P, tokens=P, verify=P, width=8, path=P, n=P + 64,
           out=P + 128, new=P + 256, anchor=P + 512):
    return lib.pbd_tree_commit(ref(pg), layers, batch, rows, start, lens, parent, tokens, verify, width, path, n, out, new,
                               anchor, None)


@pytest.mark.parametrize("call", [append, packed, tree, commit])
def test_descriptions_of_the_cache(lib, call):
    assert call(lib, None) == INV
    for kw, code in BAD_PAGES:
        if "slot_stride" in kw:
            continue
        assert call(lib, plain(**kw)) == code, kw
        assert b.pbd_last_error()
    if call is not append:
        for batch, code in ((0, INV), (-1, INV), (65536, CAP)):
            assert call(lib, plain(), batch=batch) == code
    if call in (append, commit):
        for kw in (dict(score=P), dict(slot_pos=P)):
            assert call(lib, plain(slot_stride=128, **kw)) == UNS


@pytest.mark.parametrize("call", [plan, release])
def test_tables(lib, call):
    for kw, code in [(dict(batch=0), INV), (dict(batch=65536), CAP), (dict(page=24), SHAPE), (dict(page=8), SHAPE),
                     (dict(page=8192), SHAPE), (dict(page=0), SHAPE), (dict(page=-16), SHAPE), (dict(n_pages=0), INV),
                     (dict(page=4096, n_pages=1 << 19), CAP), (dict(width=0), CAP), (dict(width=1 << 27), CAP), (dict(table=0), INV),
                     (dict(seq=0), INV), (dict(free=0), INV), (dict(n_free=0), INV)]:
        assert call(lib, **kw) == code, kw


def test_plan(lib):
    for kw in [dict(lens=0), dict(new=0), dict(start=0), dict(new_lens=0), dict(slots=0), dict(pos=0), dict(row_pos=0),
               dict(rows=-1), dict(rows=(1 << 22) + 1), dict(new_lens=P), dict(new_lens=P + 256), dict(start=P + 64),
               dict(new_lens=P + 64)]:
        assert plan(lib, **kw) == INV, kw
    assert release(lib, keep=0) == INV
    assert release(lib, keep=P) == INV


def test_append(lib):
    for kw in [dict(k=0), dict(v=0), dict(slots=0), dict(pos=0), dict(rope=0), dict(q=0), dict(q_out=0), dict(q=0, q_out=0),
               dict(rows=-1), dict(rows=(1 << 22) + 1), dict(rope_len=0), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(stride=255), dict(stride=258), dict(stride=252), dict(q=P + 4), dict(k=P + 4),
               dict(v=P + 8), dict(rope=P + 8), dict(q_out=P + 4), dict(qn=P + 2), dict(kn=P + 2)]:
        assert append(lib, plain(), **kw) == INV, kw
    assert append(lib, plain(page_size=4096, n_pages=1 << 19)) == CAP
    assert append(lib, plain(), rows=0) == b.PBD_OK


@pytest.mark.parametrize("call", [packed, tree])
def test_attention(lib, call):
    for kw, code in [(dict(q=0), INV), (dict(lens=0), INV), (dict(start=0), INV), (dict(out=0), INV), (dict(ws=0), INV),
                     (dict(q=P + 4), INV), (dict(out=P + 8), INV), (dict(ws=P + 8), INV), (dict(stride=248), INV),
                     (dict(stride=260), INV), (dict(max_len=0), INV), (dict(max_len=129), CAP), (dict(scale=0.0), INV),
                     (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(n=100), CAP), (dict(rows=0), INV),
                     (dict(rows=(1 << 22) + 1), INV), (dict(out=P), INV), (dict(lse=P), INV)]:
        assert call(lib, plain(), **kw) == code, kw
    assert call(lib, plain(n_q_heads=256, n_kv_heads=256), stride=1 << 14, rows=1 << 22) == CAP
    size = b.pbd_packed_attention_workspace_bytes if call is packed else b.pbd_tree_attention_workspace_bytes
    assert size(plain(), 2, 5, 0) == size(plain(), 2, 5, 129) == size(plain(), 2, 0, 128) == 0
    assert size(plain(), 2, 5, 128) > 0
    wide = plain(table_width=1 << 10)
    assert size(wide, 1, 2, 1 << 15) > 2 * 4 * 64 * 4 * 8


def test_tree(lib):
    assert tree(lib, plain(), mask=0) == INV
    assert tree(lib, plain(), mask=P + 4) == INV
    for kw, code in [(dict(batch=0), INV), (dict(batch=65536), CAP), (dict(rows=0), INV), (dict(start=0), INV), (dict(parent=0), INV),
                     (dict(mask=0), INV), (dict(mask=P + 4), INV), (dict(pos=0), INV), (dict(row_pos=0), INV)]:
        assert layout(lib, **kw) == code, kw
    for kw, code in [(dict(layers=0), INV), (dict(layers=1 << 23), INV), (dict(rows=0), INV), (dict(width=0), INV),
                     (dict(width=(1 << 20) + 1), INV), (dict(start=0), INV), (dict(lens=0), INV), (dict(parent=0), INV), (dict(tokens=0), INV),
                     (dict(verify=0), INV), (dict(path=0), INV), (dict(n=0), INV), (dict(out=0), INV), (dict(new=0), INV),
                     (dict(new=P), INV), (dict(out=P), INV), (dict(anchor=P + 256), INV)]:
        assert commit(lib, plain(), **kw) == code, kw
    assert commit(lib, plain(layer_stride=100), layers=2) == INV


def test_binding_refuses_host_tensors_and_wrong_types():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    k = torch.zeros(4, 2, 16 * 64, dtype=torch.bfloat16)
    pg = b.make_pages(k, k.clone(), i(2, 2), n_q_heads=4, head_dim=64)
    bf = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    f = torch.zeros(5, 256)
    ws = torch.zeros(4096, dtype=torch.uint8)
    rope = torch.zeros(9, 32, 2)
    mask = torch.zeros(5, dtype=torch.int64)
    ok = [lambda: b.pbd_page_plan(i(2, 3), i(2), i(9), i(1), i(2), i(2), 16, i(3), i(5), i(5), i(2)),
          lambda: b.pbd_page_release(i(2, 3), i(2), i(9), i(1), i(2), 16),
          lambda: b.pbd_paged_append_rows(pg, f[:, :128], f[:, 128:], i(5), i(5), rope),
          lambda: b.pbd_packed_attention(pg, bf, i(3), i(2), 32, bf, ws),
          lambda: b.pbd_tree_attention(pg, bf, i(3), i(2), mask, 32, bf, ws),
          lambda: b.pbd_tree_layout(i(3), i(5), mask),
          lambda: b.pbd_tree_commit(pg, i(3), i(2), i(5), i(5), i(5), i(2, 6), i(2), i(2, 6), i(2))]
    for call in ok:
        with pytest.raises(b.PbdError, match="on a GPU"):
            call()
    bad = [lambda: b.pbd_page_plan(i(3, 3), i(2), i(9), i(1), i(2), i(2), 16, i(3), i(5), i(5), i(2)),
           lambda: b.pbd_page_plan(i(2, 3), i(2), i(9), i(1), i(2), i(2), 16, i(2), i(5), i(5), i(2)),
           lambda: b.pbd_page_plan(i(2, 3), i(2), i(9), i(1), i(2), i(2), 16, i(3), i(4), i(5), i(2)),
           lambda: b.pbd_page_plan(i(2, 3).long(), i(2), i(9), i(1), i(2), i(2), 16, i(3), i(5), i(5), i(2)),
           lambda: b.pbd_page_release(i(3, 3), i(2), i(9), i(1), i(2), 16),
           lambda: b.pbd_paged_append_rows(pg, f[:, :128], f[:, 128:], i(4), i(5), rope),
           lambda: b.pbd_paged_append_rows(pg, f[:, :64], f[:, 128:], i(5), i(5), rope),
           lambda: b.pbd_paged_append_rows(pg, f[:, :128].bfloat16(), f[:, 128:], i(5), i(5), rope),
           lambda: b.pbd_paged_append_rows(pg, f[:, :128], f[:, 128:], i(5), i(5), rope, q=f, q_out=f),
           lambda: b.pbd_packed_attention(pg, bf.float(), i(3), i(2), 32, bf, ws),
           lambda: b.pbd_packed_attention(pg, bf, i(4), i(2), 32, bf, ws),
           lambda: b.pbd_packed_attention(pg, bf, i(4), i(3), 32, bf, ws),
           lambda: b.pbd_packed_attention(pg, bf, i(3), i(2), 32, bf.float(), ws),
           lambda: b.pbd_packed_attention(pg, bf.transpose(1, 2).contiguous().transpose(1, 2), i(3), i(2), 32, bf, ws),
           lambda: b.pbd_tree_attention(pg, bf, i(3), i(2), None, 32, bf, ws),
           lambda: b.pbd_tree_attention(pg, bf, i(3), i(2), mask[:4], 32, bf, ws),
           lambda: b.pbd_tree_attention(pg, bf, i(3), i(2), i(5), 32, bf, ws),
           lambda: b.pbd_tree_layout(i(3), i(5), mask[:4]),
           lambda: b.pbd_tree_commit(pg, i(4), i(3), i(5), i(5), i(5), i(3, 6), i(3), i(3, 6), i(3)),
           lambda: b.pbd_tree_commit(pg, i(3), i(2), i(5), i(5), i(5), i(2, 6), i(2), i(2, 5), i(2))]
    for n, call in enumerate(bad):
        with pytest.raises(b.PbdError, match="must|fewer"):
            call()


def test_the_plain_allocator_by_hand():
    t = rr.Tables([[7, -1, -1], [3, 4, -1], [-1, -1, -1]], [1, 2, 0], [0, 1, 2, 5, -1, -1, -1, -1], 4, 16)
    r = t.plan([10, 20, 0], [30, 0, 40], [10, 25, 0], 71)
    # the first takes the top two; the third needs three and finds two
    assert t.table == [[7, 5, 2], [3, 4, -1], [-1, -1, -1]] and t.n_free == 2 and r["status"] == 1
    assert r["row_start"] == [0, 30, 30, 70] and r["new_lens"] == [40, 20, 0]
    assert r["slot_map"][:7] == [7 * 16 + 10 + i for i in range(6)] + [5 * 16] and r["slot_map"][30:] == [-1] * 41
    assert r["row_seq"] == [0] * 30 + [2] * 40 + [-1] and r["row_pos"][29:31] == [39, 0]
    assert t.release([10, 3, 0]) == 0
    assert t.free[:5] == [0, 1, 4, 2, 5] and t.table == [[7, -1, -1], [3, -1, -1], [-1, -1, -1]] and t.seq_pages == [1, 1, 0]
