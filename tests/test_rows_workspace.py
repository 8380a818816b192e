"""Workspaces of the attentions of packed rows, on the host: their sizes for batches that shrink, and the bound over all."""
import random

import pytest

from paper_2607_12422_amd import binding as b
from test_paged_abi import lib, pages  # noqa: F401

SIZES = (b.pbd_packed_attention_workspace_bytes, b.pbd_tree_attention_workspace_bytes)


def cache(n_q, n_kv, hd, dtype=1, width=1 << 14):
    return pages(dtype=dtype, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd, page_size=16, page_stride=n_kv * 16 * hd,
                 head_stride=16 * hd, table_width=width, n_pages=1 << 20, score=0, slot_pos=0)


@pytest.mark.parametrize("size", SIZES)
def test_smaller_batches_may_need_more_and_none_more_than_the_bound(lib, size):  # noqa: F811
    c = cache(16, 8, 128)
    sizes = [size(c, n, 33 * n, 8192) for n in (32, 8, 1)]
    assert sizes[1] > sizes[0] and all(0 < s <= b.PBD_ROWS_WORKSPACE_MAX for s in sizes)


@pytest.mark.parametrize("size", SIZES)
def test_the_bound_holds_for_any_sizes(lib, size):  # noqa: F811
    rng = random.Random(1)
    most = 0
    for n in range(6000):
        n_kv, hd, dtype = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([64, 128]), rng.choice([0, 1])
        group = rng.choice([g for g in (1, 2, 3, 4, 5, 8, 17, 80) if n_kv * g * hd <= 16384])
        c = cache(n_kv * group, n_kv, hd, dtype)
        batch = int(2 ** rng.uniform(0, 12))
        rows = int(2 ** rng.uniform(0, 15)) if n % 2 else batch * rng.randint(1, 64)
        got = size(c, batch, rows, int(2 ** rng.uniform(0, 18)))
        assert 0 < got <= b.PBD_ROWS_WORKSPACE_MAX, (batch, rows, b.pbd_last_error())
        most = max(most, got)
    assert most > 1 << 24


def test_the_header_says_the_same():
    import os
    with open(os.path.join(os.path.dirname(b.__file__), "..", "include", "pbd.h")) as f:
        assert "#define PBD_ROWS_WORKSPACE_MAX ((size_t)48 << 20)" in f.read()
    assert b.PBD_ROWS_WORKSPACE_MAX == 48 << 20
