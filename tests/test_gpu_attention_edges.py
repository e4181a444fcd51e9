"""A decoder's attention at its edges: many queries on one head of the cache,
lengths far past the page table, some places far ahead of a long rest,
scores past fp32's range, scales of any size; the scales of appended heads."""
import math

import pytest
import torch

from paper_2109_03513_gb300 import esb
from test_gpu_attention import APPENDS, BF, FL, cached64, check_attention, i32, ints, make_cache, tables, turn64
from test_gpu_lm import TYPES, U, close, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


# More tiles of a sequence than a thread sums by itself: 8 of 8 to 32 rows.
@pytest.mark.parametrize("lens,heads,group,d", [([50, 0, 133], 1, 72, 256), ([33, 70], 1, 136, 256), ([90, 1, 20], 2, 136, 128), ([40, 61], 1, 264, 64),
                                                ([300], 1, 600, 64), ([17 + i % 40 for i in range(200)], 1, 72, 256)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_queries_on_one_head(lens, heads, group, d, dtype):
    page, seqs = 16, len(lens)
    pages = sum(-(-n // page) for n in lens) + 1
    c, t = make_cache(pages, heads, page, d, 2, 2, 5), tables(lens, page, pages, 7)
    q = rand((seqs, heads * group * d), 8, dtype)
    out = torch.full_like(q, 7.0)
    _, lse = esb.esb_cache_attention(q, c, i32(lens), t, out=out, want_lse=True)
    pick = list(range(0, seqs, max(1, seqs // 3)))
    check_attention(q[pick], c, i32(lens)[pick], t[pick], out[pick], lse[pick])
    # the same rows as sequences of one query each
    out2 = torch.full_like(q, 7.0)
    _, lse2 = esb.esb_cache_attention(q, c, i32(lens), t, starts=i32(list(range(seqs + 1))), out=out2, want_lse=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("m", [1, 3, 20])
@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_far_past_the_page_table(m, dtype):
    # their last places are not held, up to the largest length; a window over them sees nothing
    heads, group, d, page = 2, 3, 64, 16
    lens = i32([(1 << 31) - 1, 100, (1 << 31) - 40, (1 << 30) + 5, 161])
    c = make_cache(50, heads, page, d, 2, 2, 5)
    t = ints(0, 50, (5, 10), 6, torch.int32)
    q = rand((5 * m, heads * group * d), 8, dtype)
    starts = None if m == 1 else i32([m * i for i in range(6)])
    for window in (0, 1, 40, (1 << 31) - 1):
        out, lse = esb.esb_cache_attention(q, c, lens, t, starts=starts, window=window, want_lse=True)
        check_attention(q, c, lens, t, out, lse, starts=starts, window=window)
        if window in (1, 40):
            for i in (0, 2, 3):
                assert (out[m * i:m * (i + 1)] == 0).all()


LN2 = math.log(2.0)
AHEAD = [(4096, 14.0, 1.0), (4096, 18.0, 1.0), (131072, 10.0, 1.0), (131072, 14.0, 1.0), (131072, 17.0, 1.0), (131072, 20.0, 1.0),
         (131072, 17 * LN2 - math.log(1.3), 0.0), (131072, 20 * LN2 - math.log(1.3), 0.0), (131072, 25.05 * LN2, 0.0)]


@pytest.mark.parametrize("n,gap,spread", AHEAD)
@pytest.mark.parametrize("d,group,kk,vk", [(64, 2, 2, 2), (64, 20, 0, 2), (128, 4, 2, 2), (128, 12, 2, 1), (256, 1, 2, 2), (256, 12, 1, 3)])
@pytest.mark.parametrize("dtype", [FL, BF])
def test_a_few_places_far_ahead_of_the_others(n, gap, spread, d, group, kk, vk, dtype):
    # The first places (some for each warp of a block) score `gap` more than the rest, and have zero codes in half of their
    # values: what stands there is the rest's.  Scores are one product each, so that they are exact but for a few roundings.
    page, seqs = 64, 700
    k = torch.zeros((n, d), device="cuda")
    k[:, 0] = spread * rand((n,), 1) + 0.5
    v = torch.exp(0.3 * rand((n, 1), 2)).expand(n, d).clone()
    first = torch.arange(0, 128, 16, device="cuda")
    k[first, 0] = gap + 0.5
    v[first, :d // 2] = 0
    c = esb.kv_cache(n // page, 1, page, d, esb.Fmt(4, kk), esb.Fmt(4, vk))
    esb.esb_cache_append(c, k, v, torch.arange(n, device="cuda"))
    # sequences that share the pages: enough of them that a tile's work is one block's, or two blocks'
    t = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    q = torch.zeros((seqs, group, d), dtype=dtype, device="cuda")
    q[:, :, 0] = 1
    out, lse = esb.esb_cache_attention(q.flatten(1), c, i32([n] * seqs), t, scale=1.0, out=torch.empty((seqs, group * d), device="cuda"), want_lse=True)
    at = torch.arange(n // page, device="cuda")
    (k64, _), (v64, vs) = cached64(c, "k", at), cached64(c, "v", at)
    s, v64, vs = k64[0, :, 0], v64[0], vs[0]
    mx = s.max()
    e = torch.exp(s - mx)
    pr = (e / e.sum())[:, None]
    want = (pr * v64).sum(0)
    # a weight: a product and a few sums of fp32 numbers as large as the score and the largest one, and 2^x
    eta = (8 * U * (s.abs() + mx.abs()) + 2.0 ** -21)[:, None]
    # its own roundings, as documented: 11 (22) bits, and a part of the query's largest weight
    bits, floor = (2.0 ** -11, 2.0 ** -32) if dtype == BF else (2.0 ** -22, 2.0 ** -43)
    # a block's warp adds 16 places of every 64, each time off by 2^-23; instructions', warps' and parts' sums beside that
    sums = (n / 64 + 160) * 2 * U
    bound = (pr * (eta + bits) * v64.abs()).sum(0) + floor * (pr[:, 0] * vs).max() * (v64 / vs[:, None]).abs().sum(0) + \
        want.abs() * ((pr * eta).sum() + sums) + (pr * v64.abs()).sum(0) * sums
    close(out.unflatten(1, (group, d)), want.expand(seqs, group, d), bound.expand(seqs, group, d), FL)
    wl = mx + torch.log(e.sum())
    assert (lse.double() - wl).abs().max() <= (pr * eta).sum() * 1.01 + sums + 8 * U * (wl.abs() + mx.abs())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", TYPES)
def test_scores_past_the_least_fp32_number_weigh_nothing(d, dtype):
    # such a place is the first that its warp of a block sees, or the only one, or all that a whole warp sees
    group, page, n = 2, 16, 300
    c = make_cache(19, 1, page, d, 2, 2, 3)
    x = torch.zeros((n, d), device="cuda")
    x[:] = -1.0
    away = torch.zeros(n, dtype=torch.bool, device="cuda")
    away[torch.tensor([0, 16, 17, 32, 64, 100, 128], device="cuda")] = True
    away[150:256] = True
    near = rand((n, d), 4).abs() * -1.0
    k = torch.where(away[:, None], x, near)
    esb.esb_cache_append(c, k, rand((n, d), 5), torch.arange(n, device="cuda"))
    t = torch.arange(19, dtype=torch.int32, device="cuda")[None]
    q = rand((1, group * d), 8, dtype).abs() + 0.25
    for big in (3e38, float("inf")):
        c.k_scales.view(-1)[:n][away] = big
        for length in (17, 18, 33, 65, 129, 300):
            lens = i32([length])
            out, lse = esb.esb_cache_attention(q, c, lens, t, want_lse=True)
            # the same without these places: their keys far below the others
            near_c = c._replace(k_scales=c.k_scales.clone())
            near_c.k_scales.view(-1)[:n][away] = 1e3
            check_attention(q, near_c, lens, t, out, lse)


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_past_the_largest_fp32_number_are_nan(dtype):
    group, page, d, n = 2, 16, 64, 300
    c = make_cache(19, 1, page, d, 2, 2, 3)
    k = torch.ones((n, d), device="cuda")
    k[::2] = -1.0
    esb.esb_cache_append(c, k, rand((n, d), 5), torch.arange(n, device="cuda"))
    t = torch.arange(19, dtype=torch.int32, device="cuda")[None]
    q = rand((1, group * d), 8, dtype).abs() + 0.25
    for place, seen in ((1, True), (149, True), (299, True), (150, False)):
        c2 = c._replace(k_scales=c.k_scales.clone())
        c2.k_scales.view(-1)[place] = float("inf")
        out, lse = esb.esb_cache_attention(q, c2, i32([n]), t, want_lse=True)
        assert (torch.isnan(out).all() and torch.isnan(lse).all()) if seen else (torch.isfinite(out).all() and torch.isfinite(lse).all())
    assert torch.isfinite(esb.esb_cache_attention(q, c2, i32([150]), t)[0]).all()    # and one that is not seen


@pytest.mark.parametrize("kk", [0, 2])
@pytest.mark.parametrize("dtype", TYPES)
def test_scale_of_any_finite_size(kk, dtype):
    # the scale times its unit is past fp32's range, the scores are not (nor is a query's product with codes, up to 2^28,
    # times a key's scale: those lie below 2^96)
    c = make_cache(5, 1, 16, 64, kk, 2, 3)
    t, lens = torch.arange(5, dtype=torch.int32, device="cuda")[None], i32([70])
    q = rand((1, 128), 8, dtype)
    for scale, keys in ((1e37, 2.0 ** -123), (2e36, 2.0 ** -121), (1e-28, 2.0 ** 93), (-1e34, 2.0 ** -113)):
        c2 = c._replace(k_scales=c.k_scales * keys)
        out, lse = esb.esb_cache_attention(q, c2, lens, t, scale=scale, out=torch.empty_like(q, dtype=FL), want_lse=True)
        check_attention(q, c2, lens, t, out, lse, scale=float(torch.tensor(scale)))
    # no query, no score, whatever the scale
    zero = torch.zeros_like(q)
    out, lse = esb.esb_cache_attention(zero, c, lens, t, scale=3e38, want_lse=True)
    check_attention(zero, c, lens, t, out, lse, scale=1.0)


@pytest.mark.parametrize("n,heads,d,rot,inter,page", APPENDS + [
    (40, 2, 32, 32, False, 16), (21, 3, 160, 160, False, 16), (9, 1, 224, 96, False, 16), (30, 2, 64, 32, False, 16), (5, 1, 192, 64, True, 16)])
@pytest.mark.parametrize("dtype", TYPES)
def test_scales_of_spreads_are_the_projections(n, heads, d, rot, inter, page, dtype):
    # with the spread's scale too, a head's row is the group projection's bit for bit, wherever its values lie in memory
    pages = -(-n // page)
    r = esb.rotation(rot, 3000, interleaved=inter) if rot else None
    pos = ints(0, 3000, (n,), 1)
    wide = rand((n, 2 * heads * d + 16), 2, dtype)
    for at in (0, 1):
        k, v = wide[:, at:at + heads * d], wide[:, heads * d + 8 * at:2 * heads * d + 8 * at]
        c = esb.kv_cache(pages, heads, page, d, esb.Fmt(4, 2), esb.Fmt(4, 1))
        esb.esb_cache_append(c, k, v, torch.arange(n, device="cuda"), rotation=r, positions=pos if r else None, rule=esb.ESB_SCALE_DDA)
        for x, codes, scales, f in ((k, c.k_codes, c.k_scales, c.k_fmt), (v, c.v_codes, c.v_scales, c.v_fmt)):
            h = x.double().unflatten(1, (heads, d))
            if x is k:
                h = turn64(h, r.table if r else None, pos, inter)
            want, _ = esb.esb_project_groups(h.float().flatten(0, 1), f, 0, rule=esb.ESB_SCALE_DDA)
            i = torch.arange(n, device="cuda")
            assert torch.equal(scales[i // page, :, i % page], want.scales.unflatten(0, (n, heads))[..., 0])
            assert torch.equal(codes[i // page, :, i % page], want.codes.unflatten(0, (n, heads)))
