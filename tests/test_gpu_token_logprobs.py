"""pbd_token_logprobs against a plain form in 64 bits: rows and vocabularies of
all sizes, alignments and strides, masks, ties, peaked rows, padding rows."""
import math

import pytest
import torch

from paper_2607_12422_amd import binding as pbd

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"
U = 2.0 ** -24


def plain(x, tokens, n):
    """(log probabilities, entropy, ids, their log probabilities, tolerances) in 64 bits.

    Each term exp(x - m) is off by 2 U for the difference scaled to base 2 (relative to |x - m| log2 e,
    which is at most 40 where the term matters above 2^-58), 2 U of the exponential, and a sum of V terms
    rounds at most V / 256 + 40 times below it (a thread adds V / 256 of them): rel = (V / 256 + 160) U of
    S' and of T.  log(1 + S') then is off by rel S' / (1 + S') <= rel log(1 + S') and U of itself; x - m by U.
    The entropy's quotient T / (1 + S') takes rel of T and of 1 + S'."""
    V = x.shape[1]
    x = x.double()
    lp, H, ids, best, tol_lp, tol_H, tol_best = [], [], [], [], [], [], []
    for row, t in zip(x, tokens):
        m = row.max()
        if m == -math.inf:
            lp.append(-math.inf)
            H.append(0.0)
            ids.append([-1] * n)
            best.append([-math.inf] * n)
            tol_lp.append(0.0), tol_H.append(0.0), tol_best.append([0.0] * n)
            continue
        i = int(row.argmax())
        d = row - m
        e = torch.exp(d)
        e[i] = 0.0
        s = e.sum()
        lz = float(torch.log1p(s))
        T = float(torch.where(e > 0, e * d, torch.zeros_like(d)).sum())
        H.append(lz - T / (1 + float(s)))
        rel = (V / 256 + 160) * U
        tol_H.append(3 * rel * H[-1] + 1e-37)
        lp.append(float(d[t]) - lz if t >= 0 else 0.0)
        tol_lp.append(2 * rel * lz + 4 * U * abs(float(d[t])) + 1e-37 if t >= 0 and d[t] > -math.inf else 0.0)
        order = torch.sort(row, descending=True, stable=True).indices[:n]
        order = [int(j) for j in order if row[j] > -math.inf]
        ids.append(order + [-1] * (n - len(order)))
        best.append([float(d[j]) - lz for j in order] + [-math.inf] * (n - len(order)))
        tol_best.append([2 * rel * lz + 4 * U * abs(float(d[j])) + 1e-37 for j in order] + [0.0] * (n - len(order)))
    return lp, H, ids, best, tol_lp, tol_H, tol_best


def near(got, want, tol):
    want, tol = torch.tensor(want, dtype=torch.float64), torch.tensor(tol, dtype=torch.float64)
    got = got.double().cpu()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    err = (got - want).abs()[~inf]
    assert torch.all(err <= tol[~inf]), (err - tol[~inf]).max()


def check(x, tokens, n, dx=None, skip=()):
    """x: the values [rows][vocab] on the CPU; dx: the device tensor that holds them."""
    dx = x.to(DEV) if dx is None else dx
    R, V = x.shape
    f = dict(device=DEV)
    out = dict(logprob=torch.full((R,), 77.0, **f), entropy=torch.full((R,), 77.0, **f),
               top_ids=torch.full((R, n), 77, dtype=torch.int32, **f) if n else None,
               top_logprobs=torch.full((R, n), 77.0, **f) if n else None)
    status = torch.zeros(1, dtype=torch.int32, **f)
    size = pbd.pbd_token_logprobs_workspace_bytes(R, V, n)
    assert size > 0
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, **f)
    pbd.pbd_token_logprobs(dx, torch.tensor(tokens, dtype=torch.int32, **f), out["logprob"], ws, entropy=out["entropy"],
                           top_ids=out["top_ids"], top_logprobs=out["top_logprobs"], status=status)
    torch.cuda.synchronize()
    lp, H, ids, best, tl, th, tb = plain(x, [min(t, V - 1) for t in tokens], n)
    live = [r for r in range(R) if r not in skip]
    near(out["logprob"][live], [lp[r] for r in live], [tl[r] for r in live])
    near(out["entropy"][live], [H[r] for r in live], [th[r] for r in live])
    if n:
        assert out["top_ids"][live].tolist() == [ids[r] for r in live]
        near(out["top_logprobs"][live], [best[r] for r in live], [tb[r] for r in live])
    for r in skip:
        assert all(torch.all(t[r] == 77) for t in out.values() if t is not None)
    return out, int(status)


def logits(R, V, dtype=F32, seed=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(R, V, generator=g) * spread).to(dtype)
    return x, torch.randint(0, V, (R,), generator=g).tolist()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [1, 2, 7, 16, 255, 257, 1000, 4096, 8191, 8192, 8193, 50001, 151936])
def test_vocabularies(V, dtype):
    x, t = logits(3, V, dtype, seed=V)
    for n in (0, 1, 5, 32):
        out, status = check(x, t, n)
        assert status == 0


@pytest.mark.parametrize("R", [1, 2, 17, 100, 700])
def test_rows(R):
    x, t = logits(R, 20011, BF if R % 2 else F32, seed=R)
    check(x, t, 20)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("first,pad", [(0, 1), (1, 0), (3, 4), (5, 2), (7, 0), (8, 8)])
def test_alignments(first, pad, dtype):
    """Rows that begin anywhere; what lies around them may be anything."""
    x, t = logits(5, 9001, dtype, seed=first)
    buf = torch.full((5, first + 9001 + pad), math.nan, dtype=dtype, device=DEV)
    buf[:, first: first + 9001] = x.to(DEV)
    check(x, t, 12, buf[:, first: first + 9001])


@pytest.mark.parametrize("dtype", [F32, BF])
def test_masked_rows(dtype):
    """Masked tokens, rows with few tokens left, one, none; masks of the type's lowest value."""
    x, t = logits(7, 20000, dtype)
    g = torch.Generator().manual_seed(3)
    x[0][torch.rand(20000, generator=g) < 0.7] = -math.inf
    x[1, 5:] = -math.inf
    x[2, :] = -math.inf
    x[2, 12345] = 2.0
    x[3, :] = -math.inf
    x[4, 100:] = torch.finfo(dtype).min
    x[5, :] = torch.finfo(dtype).min
    x[6, :-1] = -math.inf
    t[2], t[4] = 12345, 3
    check(x, t, 20)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_ties(dtype):
    """All equal, few values, equal in pairs, and runs that ascend and descend along the row."""
    V = 30000
    x = torch.zeros(6, V)
    x[1] = torch.randint(0, 3, (V,), generator=torch.Generator().manual_seed(1)).float()
    x[2] = torch.arange(V).div(2, rounding_mode="floor") * 1e-3
    x[3] = torch.arange(V) * 1e-3
    x[4] = -torch.arange(V) * 1e-3
    x[5, ::2] = -0.0
    x = x.to(dtype)
    for n in (1, 20, 32):
        check(x, [0, 1, 2, V - 1, 0, 7], n)


def test_the_largest_in_one_thread():
    """The most likely tokens where one thread of the kernel has them all, and in one contiguous run."""
    for step in (1, 4, 8, 1024, 8192):
        x, t = logits(1, 80000, spread=0.1)
        at = torch.arange(40) * step
        at = at[at < 80000]
        x[0, at] = torch.arange(len(at)) * 0.01 + 5
        check(x, t, 32)


def test_peaked_rows_keep_their_precision():
    """One token with nearly all of the mass: values near zero, whose relative error is held."""
    x = torch.full((6, 151936), -30.0)
    for r, top in enumerate((-20.0, -10.0, 0.0, 10.0, 40.0, 90.0)):
        x[r, 77777] = top
    x[5] += torch.randn(151936, generator=torch.Generator().manual_seed(0))
    check(x, [77777] * 6, 3)


def test_nan_and_infinity():
    x, t = logits(4, 9000)
    x[1, 5000] = math.nan
    x[2, 100] = math.inf
    x[3, :] = math.nan
    R, V, n = 4, 9000, 4
    f = dict(device=DEV)
    lp, H = torch.zeros(R, **f), torch.zeros(R, **f)
    ids, best = torch.zeros(R, n, dtype=torch.int32, **f), torch.zeros(R, n, **f)
    ws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(R, V, n), dtype=torch.uint8, **f)
    pbd.pbd_token_logprobs(x.to(DEV), torch.tensor(t, dtype=torch.int32, **f), lp, ws, entropy=H, top_ids=ids,
                           top_logprobs=best)
    assert torch.isnan(lp).tolist() == [False, True, True, True]
    assert torch.isnan(H).tolist() == [False, True, True, True]
    assert torch.isnan(best).all(1).tolist() == [False, True, True, False]
    clean = torch.where(torch.isnan(x), -math.inf, x)
    want = torch.sort(clean, dim=1, descending=True, stable=True).indices[:, :n].tolist()
    assert ids.tolist() == want[:3] + [[-1] * n]


def test_padding_and_bad_tokens_skip_the_row():
    x, t = logits(6, 5000)
    t[1] = -1
    out, status = check(x, t, 5, skip=(1,))
    assert status == 0
    t[3], t[4] = 5000, -2
    out, status = check(x, t, 5, skip=(1, 3, 4))
    assert status == pbd.PBD_STATUS_TOKEN


def test_without_tokens():
    x, _ = logits(3, 5000)
    H = torch.zeros(3, device=DEV)
    ws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(3, 5000, 0), dtype=torch.uint8, device=DEV)
    pbd.pbd_token_logprobs(x.to(DEV), None, None, ws, entropy=H)
    _, want, _, _, _, tol, _ = plain(x, [0] * 3, 0)
    near(H, want, tol)


def test_three_dimensions_and_bitwise_again():
    x, t = logits(12, 151936, BF)
    a, _ = check(x, t, 20, x.to(DEV))
    b, _ = check(x, t, 20, x.to(DEV).view(4, 3, -1))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_captured_and_replayed():
    f = dict(device=DEV)
    x, t = logits(17, 30000)
    dx, dt = x.to(DEV), torch.tensor(t, dtype=torch.int32, **f)
    lp, ids, best = torch.zeros(17, **f), torch.zeros(17, 5, dtype=torch.int32, **f), torch.zeros(17, 5, **f)
    ws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(17, 30000, 5), dtype=torch.uint8, **f)
    args = (dx, dt, lp, ws)
    pbd.pbd_token_logprobs(*args, top_ids=ids, top_logprobs=best)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pbd.pbd_token_logprobs(*args, top_ids=ids, top_logprobs=best)
    for seed in (1, 2, 3):
        y, t = logits(17, 30000, seed=seed)
        dx.copy_(y)
        dt.copy_(torch.tensor(t, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want_lp, _, want_ids, want_best, tl, _, tb = plain(y, t, 5)
        near(lp, want_lp, tl)
        near(best, want_best, tb)
        assert ids.tolist() == want_ids


def test_rows_past_32_bits():
    """Rows 2^29 elements apart, the last one 2^31 from the first."""
    x, _ = logits(5, 1001, BF, seed=29)
    far = torch.empty(4 * 2 ** 29 + 1001, dtype=BF, device=DEV).as_strided((5, 1001), (2 ** 29, 1))
    far.copy_(x)
    check(x, [3, 999, -1, 0, 1000], 7, dx=far, skip=(2,))


MASKS = [-1e6, -1.2e6, -1e9, -4e9, -1e10, -1e12, -1e15, -1e20, -1e29, -2e30, -3e38]


def masked_by(mask, R, V, dtype):
    """Rows with a finite mask: a few tokens left, early, late, in the middle; half of them; none; the first tiles."""
    x, t = logits(R, V, dtype, seed=7)
    for r in range(R):
        live = {0: [0, 1, 2], 1: [V - 3, V - 1], 2: [9000, 9001, 9007], 3: range(0, V, 2), 4: [], 5: range(9 * V // 10, V),
                6: range(V // 100)}[r % 7]
        live = torch.tensor(list(live), dtype=torch.long)
        row = torch.full((V,), mask).to(dtype)
        row[live] = x[r, live]
        x[r] = row
        if len(live) and r % 14 < 11:
            t[r] = int(live[t[r] % len(live)])
    return x, t


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("mask", MASKS)
def test_finite_masks(mask, dtype):
    """Masks that are numbers, as a constrained vocabulary has them, whole tiles and rows of them among the rest."""
    x, t = masked_by(mask, 14, 40000, dtype)
    check(x, t, 5)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("mask", MASKS)
def test_finite_masks_of_many_rows(mask, dtype):
    """The same where one work-group takes a whole row, tile after tile."""
    x, t = masked_by(mask, 14, 40000, dtype)
    many = x.to(DEV).repeat(40, 1)
    a, _ = check(many[:14].cpu(), t, 5)
    f = dict(device=DEV)
    lp, H, best = torch.zeros(560, **f), torch.zeros(560, **f), torch.zeros(560, 5, **f)
    ids = torch.zeros(560, 5, dtype=torch.int32, **f)
    ws = torch.empty(pbd.pbd_token_logprobs_workspace_bytes(560, 40000, 5), dtype=torch.uint8, **f)
    pbd.pbd_token_logprobs(many, torch.tensor(t * 40, dtype=torch.int32, **f), lp, ws, entropy=H, top_ids=ids,
                           top_logprobs=best)
    want_lp, want_H, want_ids, want_best, tl, th, tb = plain(x, t, 5)
    for i in range(40):
        at = slice(14 * i, 14 * i + 14)
        near(lp[at], want_lp, tl)
        near(H[at], want_H, th)
        near(best[at], want_best, tb)
        assert ids[at].tolist() == want_ids


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("size", [1e4, 2.0 ** 20, 1e9, 4e9, 1e20, 1e29, 3e38])
def test_large_logits(size, dtype):
    """Equal rows of a size, and rows that reach it once, in both signs."""
    x = torch.full((6, 30000), size)
    x[1] = -size
    x[2] = 0.0
    x[2, 20000] = size
    x[3] = torch.linspace(-size, size, 30000, dtype=torch.float64).float()
    x[4] = -x[3]
    x[5, ::3] = -size
    check(x.to(dtype), [5, 6, 20000, 29999, 0, 1], 8)


@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 16, 2.0 ** 18, 2.0 ** 20, 2.0 ** 22, 2.0 ** 30])
def test_maxima_that_cross_a_size(size):
    """Maxima that rise and fall from tile to tile past a power of two, in both signs, a row to a work-group."""
    V, tile = 50000, 8192
    g = torch.Generator().manual_seed(5)
    step = max(2.0 ** -8, size * 2.0 ** -22)
    base = (torch.arange(V) // tile).double()
    rows = []
    for sign in (1.0, -1.0):
        for slope in (1.0, -1.0):
            noise = torch.rand(2, V, generator=g, dtype=torch.float64) * -4.0
            rows.append(sign * size + slope * (base - 3.0) + noise)
    x = torch.cat(rows).div(step).round().mul(step).float()
    x = x.repeat(65, 1)
    check(x, torch.randint(0, V, (520,), generator=g).tolist(), 4)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("R", [1, 3])
def test_ties_over_many_parts(R, dtype):
    """A row of equal logits in more parts than the join has room to rank at once."""
    x = torch.full((R, 151936), 0.5, dtype=dtype)
    x[R - 1, :3] = -math.inf
    check(x, [7] * R, 32)
