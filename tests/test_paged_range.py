"""Prefill attention over the paged cache where values of very different size meet, against the model in 64 bits: what a row does not
see or gives no weight must not cost the values that it does see their bits."""
import math

import pytest
import torch

import paged_model as M
import test_paged as P

pytestmark = pytest.mark.gpu
gpu = P.gpu


def _expected(w, rows, window, scale, q, lens=None):
    """Outputs in 64 bits and what each may be off by, the last rows[b] tokens of every sequence, one after the other.

    Once eps / 2 of the value (or half the type's smallest step).  A weight: 2 * 136 * 2^-24 of the sum of magnitudes behind the
    score (128 products, eight factors, numerator and denominator), 2 * 2^-11 for its fp16 rounding and the sum's, 2 * 64 * 2^-24 for
    sums with a rescaling per block.  A weight below fp16's normal range is off by half of fp16's smallest step, 2^-25, with the
    row's largest at 2^8 or more: 2^-33 of the sum of the weights; but where it rounds to nothing, by itself."""
    now, out, tol, at = M.Snapshot(w.cache), [], [], 0
    lens = w.lens if lens is None else lens
    eps, G = torch.finfo(w.dtype).eps / 2, w.Hq // w.H
    for b, n in enumerate(rows):
        if n == 0:
            continue
        k, v = now.held(w.table[b], w.tails[b], lens[b])
        pos, j = torch.arange(lens[b] - n, lens[b])[:, None], torch.arange(lens[b])
        seen = j <= pos
        if window:
            seen &= j > pos - window
        for g in range(w.Hq):
            x = q[at:at + n, g].double()
            kk, vv = k[:, g // G], v[:, g // G]
            s = torch.where(seen, x @ kk.t() * scale, torch.full((), -math.inf, dtype=torch.float64))
            spread = torch.where(seen, x.abs() @ kk.abs().t() * abs(scale), torch.zeros((), dtype=torch.float64)).amax(1, keepdim=True)
            p = torch.softmax(s, dim=-1)
            o, size, faint = p @ vv, p @ vv.abs(), p.clamp(max=2.0 ** -33) @ vv.abs()
            share = 2 * 136 * 2.0 ** -24 * spread + 2 * 2.0 ** -11 + 2 * 64 * 2.0 ** -24
            off = share * size + faint
            out.append(o)
            tol.append(off + eps * (o.abs() + off) + (2.0 ** -25 if w.dtype is torch.float16 else 2.0 ** -134))
        at += n
    heads = lambda x: torch.cat([torch.stack(x[i:i + w.Hq], dim=1) for i in range(0, len(x), w.Hq)])  # noqa: E731
    return heads(out), heads(tol)


def _check(w, rows, q, window=0, scale=None, **kw):
    scale = 1 / math.sqrt(w.D) if scale is None else scale
    got = w.cache.attn_prefill(q.cuda(), scale, P._starts(rows), P._i32(w.lens), w.d_table, w.d_tails, window=window, **kw).cpu().double()
    want, tol = _expected(w, rows, window, scale, q)
    err = (got - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float((err / tol).max()))
    return got


def _sided(w, counts, small, sizes, turned):
    """Tokens whose keys point along a direction u where small(b, place) says so, away from it elsewhere, and whose values are sizes[0]
    times as large there, sizes[1] times elsewhere; queries along u, those of every `turned`-th token away from it."""
    n = sum(counts)
    k, v, q = w.rand(n, w.H, w.D), w.rand(n, w.H, w.D), w.rand(n, w.Hq, w.D)
    u = torch.where(w.rand(w.D) > 0, 1.0, -1.0)
    side = torch.tensor([bool(small(b, i)) for b, c in enumerate(counts) for i in range(c)])
    k = 0.5 * k + 8 * u * torch.where(side, 1.0, -1.0)[:, None, None]
    v = v * torch.where(side, sizes[0], sizes[1])[:, None, None]
    q = u + 0.1 * q
    q[::turned] *= -1
    return k.to(w.dtype), v.to(w.dtype), q.to(w.dtype)


SIZES = {torch.float16: [(2.0 ** -13, 2.0 ** 13)], torch.bfloat16: [(2.0 ** -13, 2.0 ** 13), (2.0 ** -30, 1.0), (2.0 ** -30, 2.0 ** 60)]}


@pytest.mark.parametrize("H", [1, 64], ids=["split keys", "one workgroup for all keys"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,codes", P.TYPES, ids=P.IDS)
def test_the_weight_lies_on_pages_of_small_values(gpu, dtype, codes, D, H):
    """Pages whose V scales are 2^26 and more apart, the larger ones first, between and last; keys give them no weight, or all."""
    for sizes in SIZES[dtype]:
        w = P.World(gpu, 3, H, 2 if H == 1 else 1, D, dtype, codes, 5, seed=D)
        counts = [320, 256, 192]
        large = {0: (0, 3), 1: (1, 2), 2: (2,)}
        k, v, q = _sided(w, counts, lambda b, i: i // 64 not in large[b], sizes, 5)
        w.append(counts, k, v)
        _check(w, counts, q)
        _check(w, counts, q, max_new=1)  # the other shape of the launch
        w.check()


@pytest.mark.parametrize("H", [1, 64], ids=["split keys", "one workgroup for all keys"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,codes", P.TYPES, ids=P.IDS)
def test_large_values_that_the_window_hides(gpu, dtype, codes, D, H):
    """The first block's values are 2^26 times the others'; the rows behind the window do not see them, the tile's first rows do."""
    w = P.World(gpu, 2, H, 1, D, dtype, codes, 6, seed=D + 1)
    counts = [384, 320]
    k, v, q = w.tokens(sum(counts))
    v = v.double() * 2.0 ** -13
    for at in (0, 384):
        v[at:at + 64] *= 2.0 ** 26
    w.append(counts, k, v.to(dtype))
    _check(w, counts, q, window=64)
    _check(w, counts, q, window=100, max_new=1)
    w.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_the_smallest_values_beside_an_unfinished_block(gpu, codes, D):
    """bf16 values around 2^-98, with and without an unfinished block: its unit is far above theirs."""
    for rest in (0, 22):
        w = P.World(gpu, 2, 64, 1, D, torch.bfloat16, codes, 6, seed=D + rest)
        counts = [320 + rest, 256 + rest]
        k, v, q = w.tokens(sum(counts))
        w.append(counts, k, (v.double() * 2.0 ** -98).to(torch.bfloat16))
        _check(w, counts, q)
        w.check()


@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_values_of_all_sizes_before_an_unfinished_block(gpu, codes):
    """bf16 pages of 2^110 that have no weight, in an unfinished block's workgroup whose values are small, and the other way round."""
    for sizes in ((2.0 ** -20, 2.0 ** 110), (2.0 ** 110, 2.0 ** -20)):
        w = P.World(gpu, 2, 64, 1, 64, torch.bfloat16, codes, 4, seed=7)
        counts = [150, 90]
        k, v, q = _sided(w, counts, lambda b, i: i // 64 == counts[b] // 64, sizes, 5)
        w.append(counts, k, v)
        _check(w, counts, q)
        w.check()


@pytest.mark.parametrize("dtype,codes", P.TYPES[2:], ids=P.IDS[2:])
def test_split_keys_with_values_of_all_sizes(gpu, dtype, codes):
    """Few rows over a long past, whose splits are in units 2^120 and more apart: all keys small beside an unfinished block, and pages of
    2^110 without weight before it."""
    for D, rest in ((64, 22), (128, 22), (128, 0)):
        w = P.World(gpu, 2, 1, 2, D, dtype, codes, 64, seed=D)
        counts = [64 * 61 + rest, 64 * 20 + rest]
        k, v, q = w.tokens(sum(counts))
        w.append(counts, k, (v.double() * 2.0 ** -98.5).to(dtype))
        _check(w, [3, 5], q[:8])
        w.check()
    w = P.World(gpu, 2, 1, 2, 64, dtype, codes, 64, seed=6)
    counts = [64 * 61 + 30, 64 * 20 + 10]
    k, v, q = _sided(w, counts, lambda b, i: i // 64 == counts[b] // 64, (2.0 ** -40, 2.0 ** 110), 100000)
    w.append(counts, k, v)
    _check(w, [3, 5], q[1:9])
    w.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_small_values_of_an_unfinished_block_behind_large_ones(gpu, codes, D):
    """fp16 values near the type's smallest step in the unfinished block, 2^15 in the pages, which the window or the keys leave no weight."""
    for window in (0, 8):
        w = P.World(gpu, 2, 64, 1, D, torch.float16, codes, 5, seed=D + window)
        counts = [64 * 4 + 40, 64 * 2 + 60]
        k, v, q = _sided(w, counts, lambda b, i: i // 64 == counts[b] // 64, (2.0 ** -20, 2.0 ** 13), 5)
        w.append(counts, k, v)
        _check(w, counts, q, window=window)
        w.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("codes", ["int8", "e4m3"])
def test_scores_of_minus_infinity(gpu, codes, D):
    """bf16 scores below binary32's range take no part, whether they come first or last; a row with no others is zero; one above it makes
    the row NaN.  The same from both calls."""
    for H in (1, 64):
        w = P.World(gpu, 3, H, 1, D, torch.bfloat16, codes, 4, seed=D)
        counts = [64 + 64 + 30, 128 + 20, 100]
        k, v, _ = w.tokens(sum(counts))
        q = (1 + w.rand(sum(counts), H, D).abs()).to(torch.bfloat16) * 1e20
        k = (k.double() * 1e-20).to(torch.bfloat16)
        far = torch.zeros(sum(counts), dtype=torch.bool)
        far[:64] = True             # the first block
        far[158 + 128:158 + 148] = True   # an unfinished one
        far[306:] = True            # all
        k[far] = -1e20
        w.append(counts, k, v)
        lens, args = P._i32(w.lens), (w.d_table, w.d_tails)
        got = w.cache.attn_prefill(q.cuda(), 0.1, P._starts(counts), lens, *args).cpu().double()
        assert not got[:64].any() and not got[306:].any()
        # the rows that see others too: as if the far ones were not there
        now = M.Snapshot(w.cache)
        for b, first, last in ((0, 64, 158), (1, 158, 306)):
            kk, vv = now.held(w.table[b], w.tails[b], counts[b])
            at = 158 * b
            j = torch.arange(counts[b])
            for i in range(first, last):
                seen = (j <= i - at) & ~far[at:at + counts[b]]
                s = torch.where(seen[:, None], (q[i].double() * kk).sum(-1) * 0.1, torch.full((), -math.inf, dtype=torch.float64))
                spread = torch.where(seen[:, None], (q[i].double() * kk).abs().sum(-1) * 0.1, torch.zeros((), dtype=torch.float64)).amax(0)
                p = torch.softmax(s, dim=0)
                want, size = (p[..., None] * vv).sum(0), (p[..., None] * vv.abs()).sum(0)
                faint = (p.clamp(max=2.0 ** -33)[..., None] * vv.abs()).sum(0)
                share = 2 * 136 * 2.0 ** -24 * spread[:, None] + 2 * 2.0 ** -11 + 2 * 64 * 2.0 ** -24
                off = share * size + faint
                assert bool(((got[i] - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()), (b, i)
        one = w.cache.attn_decode(q[[157, 305, 405]].cuda(), 0.1, lens, *args).cpu().double()
        few = w.cache.attn_prefill(q[[157, 305, 405]].cuda(), 0.1, P._i32([0, 1, 2, 3]), lens, *args, max_new=1).cpu().double()
        assert not one[2].any() and not few[2].any()
        # against the chunk's: a rounding to bf16 on either side, and two of weights to 11 bits, of values up to 5
        for x in (one, few):
            assert bool(((x[:2] - got[[157, 305]]).abs() <= 2.0 ** -7 * x[:2].abs() + 2.0 ** -8 * 5).all())
        up = w.cache.attn_prefill((-q).cuda(), 0.1, P._starts(counts), lens, *args)
        assert torch.isnan(up[:158]).all() and torch.isnan(up[306:]).all()
        assert torch.isnan(w.cache.attn_decode((-q[[157, 305, 405]]).cuda(), 0.1, lens, *args)).all()
