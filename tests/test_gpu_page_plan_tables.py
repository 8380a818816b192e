"""pbd_page_plan where a table holds ids that are no pages: no slot of another page comes of them."""
import pytest
import torch

from paper_2607_12422_amd import binding as pbd
from test_gpu_page_plan import DEV, i32

pytestmark = pytest.mark.gpu

PAGE, N = 16, 20


def plan(table, have, lens, new, R, status=True, n_free=6):
    free = i32(list(range(10, 10 + n_free)) + [-1] * (N - n_free))
    B = len(lens)
    out = dict(table=i32(table), seq_pages=i32(have), n_free=i32([n_free]), row_start=i32([0] * (B + 1)), row_seq=i32([0] * R),
               row_pos=i32([0] * R), slot_map=i32([-55] * R), new_lens=i32([0] * B), status=i32([0]))
    pbd.pbd_page_plan(out["table"], out["seq_pages"], free, out["n_free"], i32(lens), i32(new), PAGE, out["row_start"],
                      out["row_seq"], out["slot_map"], out["new_lens"], pos=i32(lens), row_pos=out["row_pos"],
                      status=out["status"] if status else None)
    return {n: t.tolist() for n, t in out.items()}


@pytest.mark.parametrize("rows", [50, 5000])
@pytest.mark.parametrize("bad", [-1, N, 2 ** 28 + 3, 2 ** 27, 2 ** 31 - 1, -2 ** 31, -2 ** 28 + 4])
def test_rows_of_a_bad_page_have_no_slot(bad, rows):
    """The last used page, an earlier one (which no row goes to) and one that was taken ahead; by one launch and by two."""
    table = [[3, 4, -1, -1], [5, bad, -1, -1], [bad, 6, -1, -1], [7, 8, bad, 9]]
    have, lens, new = [2, 2, 2, 4], [20, 20, 20, 30], [5, 14, 5, 25]
    r = plan(table, have, lens, new, rows)
    slots = []
    for b, (m, n) in enumerate(zip(lens, new)):
        for s in range(m, m + n):
            page = r["table"][b][s // PAGE]
            slots.append(page * PAGE + s % PAGE if 0 <= page < N else -1)
    # sequence 1 takes a page, the top of the stack
    assert r["table"][1] == [5, bad, 15, -1] and r["n_free"] == [5] and r["seq_pages"] == [2, 3, 2, 4]
    assert slots[5:5 + 12] == [-1] * 12 and slots[17:19] == [240, 241] and slots.count(-1) == 12 + 16
    assert r["slot_map"] == slots + [-1] * (rows - len(slots))
    assert r["status"] == [pbd.PBD_STATUS_PAGE] and r["new_lens"] == [25, 34, 25, 55]


def test_without_a_status_word():
    r = plan([[3, 2 ** 28 + 3]], [2], [20], [4], 6, status=False)
    assert r["slot_map"] == [-1] * 6


def test_an_append_after_such_a_plan_leaves_other_pages_alone():
    """An id of 2^28 + 3 is page 3 in 32 bits: the rows are skipped, and the status says so."""
    H, D = 2, 64
    r = plan([[1, 2 ** 28 + 3], [3, 4]], [2, 2], [20, 18], [4, 3], 8)
    assert r["status"] == [pbd.PBD_STATUS_PAGE] and r["slot_map"] == [-1] * 4 + [66, 67, 68, -1]
    k, v = (torch.full((N, H, PAGE * D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pages = pbd.make_pages(k, v, i32(r["table"]), n_q_heads=H, head_dim=D)
    x = torch.ones(8, H * D, device=DEV)
    rope = torch.zeros(64, D // 2, 2, device=DEV)
    pbd.pbd_paged_append_rows(pages, x, x, i32(r["slot_map"]), i32(r["row_pos"]), rope)
    changed = [p for p in range(N) if not bool((v[p] == 7.0).all())]
    assert changed == [4]
