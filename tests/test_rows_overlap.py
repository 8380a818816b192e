"""pbd_tree_commit's outputs that lie over an input or each other, in part too: refused on the host, before anything runs
(every work-group of a sequence reads the inputs while the first one writes)."""
import pytest

from paper_2607_12422_amd import binding as b
from test_paged_abi import INV, P, lib, pages  # noqa: F401

BATCH, ROWS, WIDTH = 3, 40, 20
IN = dict(row_start=BATCH + 1, before=BATCH, lens=BATCH, parent=ROWS, tokens=ROWS, verify=ROWS, table=4 * BATCH)
OUT = dict(path=BATCH * WIDTH, n_accepted=BATCH, out_tokens=BATCH * WIDTH, new_lens=BATCH, anchor=BATCH)


def commit(lib, at, served):  # noqa: F811
    pg = pages(score=0, slot_pos=0, table=at["table"])
    fn, before = (lib.pbd_tree_commit_served, (at["before"],)) if served else (lib.pbd_tree_commit, ())
    return fn(b.ctypes.byref(pg), 1, BATCH, ROWS, at["row_start"], *before, at["lens"], at["parent"], at["tokens"], at["verify"],
              WIDTH, at["path"], at["n_accepted"], at["out_tokens"], at["new_lens"], at["anchor"], None)


@pytest.mark.parametrize("served", [False, True])
@pytest.mark.parametrize("out", OUT)
def test_outputs_over_inputs_and_each_other(lib, out, served):  # noqa: F811
    every = dict(IN, **OUT)
    for other, n in every.items():
        if other == out or (other == "before" and not served):
            continue
        # the same place, the last element's, and one whose last element is the other's first
        for shift in (0, n - 1, 1 - every[out]):
            at = {name: P + (i << 12) for i, name in enumerate(every)}
            at[out] = at[other] + 4 * shift
            assert commit(lib, at, served) == INV, (other, shift)
            assert "overlap" in b.pbd_last_error()


def test_before_is_given(lib):  # noqa: F811
    at = {name: P + (i << 12) for i, name in enumerate(dict(IN, **OUT))}
    assert commit(lib, dict(at, before=0), True) == INV
