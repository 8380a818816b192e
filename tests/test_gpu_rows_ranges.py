"""pbd_packed_attention and pbd_tree_attention where scores or values are far from 1: what a row gets when its tile is gone
over a second time, in one part and in several."""
import math

import pytest
import torch

import paged_ref as ref
import rows_ref as rr
from paper_2607_12422_amd import binding as pbd
from test_gpu_packed_attention import BF, DEV, F32, Call

pytestmark = pytest.mark.gpu

U = ref.U


def spread(parts, D, dtype):
    """(cache, rows of each sequence): one sequence of 150 rows over as many slots, or of 40 over 3000."""
    return (ref.Cache([3000], 1, D, dtype, seed=6), [40]) if parts else (ref.Cache([150], 1, D, dtype, seed=6), [150])


def put(cache, k0):
    """Keys that are 0 but in dim 0."""
    n = cache.lens[0]
    cache.dk[0, 0, :n] = 0.0
    cache.dk[0, 0, :n, 0] = k0.to(cache.dtype)
    cache.put(0, 0, cache.dk[0, :, :n], cache.dv[0, :, :n])


def call(cache, counts, e, masks=None):
    c = Call(cache, counts, 1, masks=masks)
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 2.0 ** e
    c.dq.copy_(c.q.to(DEV))
    return c


@pytest.mark.parametrize("parts", [False, True])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_score_far_above_the_others(dtype, odd, parts):
    """Scores up to some 2^14 .. 2^37, also where the last slot's NaN, hidden from the rows before, sends their tile through
    the second pass: each row gets the mean of the highest slots that it sees.

    Scores are products of one power of two, exact, and 2^14 / 8 at least apart, so that the others' weights are 0.  Equal
    scores have equal weights, whatever the reference: n + 80 roundings of the sums, four of the quotients and factors, and in
    bf16 one of the weight, half a step; the output's own."""
    D = 64
    half = torch.finfo(dtype).eps / 2
    for e in (14, 17, 18, 20, 23, 24, 26, 28, 29, 30):
        for down in (False, True):
            cache, counts = spread(parts, D, dtype)
            n, R = cache.lens[0], counts[0]
            ramp = torch.arange(n) * 37 % 113 if parts else torch.arange(n) % 113
            k0 = 5.0 + (112 - ramp if down else ramp)    # (up to 117: products with the scale are not exact)
            if odd:
                cache.dv[0, 0, n - 1] = math.nan
            put(cache, k0)
            c = call(cache, counts, e)
            assert (c.ws.numel() > 256) == parts
            c.run()
            out, lse, v = c.out.double().cpu(), c.lse.double().cpu(), cache.dv[0, 0].double()
            for i in range(R):
                if odd and i == R - 1:
                    assert torch.isnan(out[i, 0]).all()
                    continue
                seen = k0[: n - R + i + 1].double()
                top = (seen == seen.max()).nonzero()[:, 0]
                want, size = v[top].mean(0), v[top].abs().mean(0)
                tol = want.abs() * half * 1.01 + size * ((n + 84) * U + (half * 1.01 if dtype == BF else 0.0))
                off = (out[i, 0] - want).abs()
                assert torch.all(off <= tol), (e, down, i, (off / size).max())
                s = float(seen.max()) * 2.0 ** e / 8
                assert abs(float(lse[i, 0]) - s - math.log(len(top))) <= 8 * U * s + (n + 84) * U


@pytest.mark.parametrize("parts", [False, True])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("down", [False, True])
def test_scores_one_step_apart(down, odd, parts):
    """fp32 scores past 2^31, each a step of the type above (below) the one before: in units of log2 some of two such round to
    one number.  A row gets the highest slot that it sees, or a mean of it and slots that are one step below."""
    D = 64
    for e in (33, 60, 92):
        cache, counts = spread(parts, D, F32)
        n, R = cache.lens[0], counts[0]
        step = torch.arange(n).double()
        k0 = 1.9 + (n - 1 - step if down else step) * 2.0 ** -23
        k0 = k0.float()
        assert torch.all((k0.double().diff().abs() * 2 ** 23).round() == 1)
        if odd:
            cache.dv[0, 0, n - 1] = math.nan
        put(cache, k0)
        c = call(cache, counts, e)
        assert (c.ws.numel() > 256) == parts
        c.run()
        out, v = c.out.double().cpu(), cache.dv[0, 0].double()
        for i in range(R - 1 if odd else R):
            last = 0 if down else n - R + i
            pair = v[[last, min(1, n - R + i) if down else max(0, last - 1)]]
            tol = 4 * U * pair.abs().amax(0)
            assert torch.all(out[i, 0] >= pair.amin(0) - tol) and torch.all(out[i, 0] <= pair.amax(0) + tol), (e, i)


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_query_that_is_not_finite_beside_large_scores(dtype, D, trees):
    """Rows of a tile in which another row's query is NaN, ordinary weights between scores of some thousands: the bound that
    holds without it holds with it."""
    g = torch.Generator().manual_seed(D)
    for lens, counts in (([150, 40], [60, 40]), ([3000], [40])):
        t = [rr.random_tree(n, g) for n in counts] if trees else None
        c = Call(ref.Cache(lens, 2, D, dtype, seed=7), counts, 2, trees=t)
        c.dq[3, 1, 5] = math.nan
        c.run(scale=2000.0)
        assert torch.isnan(c.out[3, 1]).all() and torch.isnan(c.lse[3, 1])
        out, lse = c.out.clone(), c.lse.clone()
        c.dq.copy_(c.q.to(DEV))
        c.run(scale=2000.0)
        c.check(scale=2000.0)
        out[3, 1], lse[3, 1] = c.out[3, 1], c.lse[3, 1]
        c.out.copy_(out)
        c.lse.copy_(lse)
        c.check(scale=2000.0)


@pytest.mark.parametrize("trees", [False, True])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("kind", ["rising", "flat", "any"])
def test_values_near_the_largest_finite_ones(kind, dtype, D, trees):
    """Values up to 2^127, of either sign or of one: a weighted mean of them is finite, however many slots share the weight
    and however far the scores rise.  The bound is the usual one, relative to the values."""
    g = torch.Generator().manual_seed(D)
    for lens, counts in (([200, 33, 1500], [64, 33, 64]), ([3000], [40]), ([9000, 700], [3, 64])):
        for e in (110, 126):
            cache = ref.Cache(lens, 1, D, dtype, seed=2)
            cache.dv = (cache.dv.float().clamp(-1.9, 1.9) * 2.0 ** e).to(dtype)
            if kind != "any":
                cache.dv = cache.dv.abs()
            for b, m in enumerate(lens):
                if kind != "any":
                    cache.dk[b, 0, :m] = 0.0
                    cache.dk[b, 0, :m, 0] = (torch.arange(m) % 200).to(dtype)
                cache.put(b, 0, cache.dk[b, :, :m], cache.dv[b, :, :m])
            c = Call(cache, counts, 2, trees=[rr.random_tree(n, g) for n in counts] if trees else None)
            if kind != "any":
                c.q = torch.zeros_like(c.q)
                c.q[..., 0] = 0.0 if kind == "flat" else 0.25
                c.dq.copy_(c.q.to(DEV))
            c.run(scale=0.5)
            assert torch.isfinite(c.out[: c.starts[-1]]).all(), (lens, e)
            c.check(scale=0.5)


@pytest.mark.parametrize("parts", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_values_under_large_scores(dtype, parts):
    """What a rounded reference leaves in the exponent, up to 2^64, reaches no value: the highest slot's values come out."""
    D = 64
    half = torch.finfo(dtype).eps / 2
    for e in (17, 24, 28, 30):
        cache, counts = spread(parts, D, dtype)
        n, R = cache.lens[0], counts[0]
        cache.dv = (cache.dv.float().clamp(-1.9, 1.9).abs() * 2.0 ** 126).to(dtype)
        put(cache, 5.0 + torch.arange(n) * 37 % 113)
        c = call(cache, counts, e)
        c.run()
        out, v = c.out.double().cpu(), cache.dv[0, 0].double()
        k0 = cache.dk[0, 0, :n, 0].double()
        for i in range(R):
            seen = k0[: n - R + i + 1]
            top = (seen == seen.max()).nonzero()[:, 0]
            want, size = v[top].mean(0), v[top].abs().mean(0)
            tol = want.abs() * half * 1.01 + size * ((n + 84) * U + (half * 1.01 if dtype == BF else 0.0))
            assert torch.all((out[i, 0] - want).abs() <= tol), (e, i)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_values_that_all_rows_see(dtype):
    """An infinite value under a weight is infinite in its dim, both signs together are NaN; other dims keep the bound."""
    for lens, counts in (([150], [40]), ([3000], [40])):
        cache = ref.Cache(lens, 1, 64, dtype, seed=3)
        n = lens[0]
        clean = cache.dv.clone()
        cache.dv[0, 0, 50, 3] = math.inf
        cache.dv[0, 0, n - 60, 4] = -math.inf
        cache.dv[0, 0, 20, 9], cache.dv[0, 0, n - 50, 9] = math.inf, -math.inf
        cache.put(0, 0, cache.dk[0, :, :n], cache.dv[0, :, :n])
        c = Call(cache, counts, 2)
        c.run()
        out = c.out.double().cpu()[: counts[0]]
        assert torch.all(out[..., 3] == math.inf) and torch.all(out[..., 4] == -math.inf) and torch.isnan(out[..., 9]).all()
        cache.dv = clean
        o, _, tol, _ = rr.attention(cache, 0, c.q[: counts[0]], c.see(0), 64 ** -0.5)
        keep = [d for d in range(64) if d not in (3, 4, 9)]
        assert torch.all((out - o).abs()[..., keep] <= tol[..., keep])


@pytest.mark.parametrize("trees", [False, True])
def test_one_workspace_for_batches_that_shrink(trees):
    """The largest batch's workspace is too small for the ones after it; one of the documented bound does for all."""
    ws = torch.full((pbd.PBD_ROWS_WORKSPACE_MAX,), 0xFF, dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(4)
    need = []
    for B in (64, 20, 5, 1):
        lens = [2000 - 7 * i for i in range(B)]
        c = Call(ref.Cache(lens, 4, 64, BF, page=64, seed=B), [33] * B, 2, max_len=2048,
                 trees=[rr.random_tree(33, g) for _ in lens] if trees else None)
        need.append(c.ws.numel())
        c.ws = ws
        c.run()
        c.check()
    assert max(need) > need[0] and max(need) <= ws.numel()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64)])
def test_parts_whose_every_score_is_infinite(dtype, D):
    """Keys that make scores of -inf along whole parts, before, between and behind the others: those slots have weight 0.
    Where a row sees nothing else it is NaN, as in fp32 arithmetic, and so is a row with a score of +inf."""
    n, R = 3000, 40
    for first, end in ((0, 1500), (700, 2000), (2500, 2960), (0, 2940)):
        cache = ref.Cache([n], 1, D, dtype, seed=5)
        cache.dk[0, 0, first:end, 0] = -math.inf
        cache.put(0, 0, cache.dk[0, :, :n], cache.dv[0, :, :n])
        c = Call(cache, [R], 2)
        assert c.ws.numel() > 256
        c.q[..., 0] = c.q[..., 0].abs() + 0.5
        c.dq.copy_(c.q.to(DEV))
        c.run()
        out, lse = c.out.double().cpu()[:R], c.lse.double().cpu()[:R]
        see = rr.causal(R, n)
        see[:, first:end] = False
        cache.dk[0, 0, first:end, 0] = 0.0
        o, s, tol, s_tol = rr.attention(cache, 0, c.q[:R], see, D ** -0.5)
        assert torch.all((out - o).abs() <= tol), (first, end)
        assert torch.all((lse - s).abs() <= s_tol)
    cache.dk[0, 0, :, 0] = -math.inf
    cache.dk[0, 0, n - 10, 0] = math.inf
    cache.put(0, 0, cache.dk[0, :, :n], cache.dv[0, :, :n])
    c = Call(cache, [R], 2)
    c.q[..., 0] = 1.0
    c.dq.copy_(c.q.to(DEV))
    c.run()
    assert torch.isnan(c.out[:R]).all() and torch.all(c.lse[: R - 10] == -math.inf) and torch.isnan(c.lse[R - 10: R]).all()
