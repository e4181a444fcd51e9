"""A decoder's attention against plain 64-bit implementations: norms of heads
with rotation and their gradient, appending to a 4-bit cache (bit for bit with
the group projection), attention over it.  Tolerances count the roundings on
the way (u = 2^-24 for fp32), as written beside them."""
import math

import pytest
import torch

import oracle as o
from paper_2109_03513_gb300 import esb
from test_gpu_lm import HALF, TYPES, U, close, rand

pytestmark = pytest.mark.gpu

F64 = torch.float64
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def ints(lo, hi, shape, seed, dtype=torch.int64):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=dtype)


def turn64(x, table, pos, inter, back=False):
    """Heads (tokens, heads, d) in 64 bits, turned by the table's angles of each token."""
    if table is None:
        return x
    rot = table.shape[1]
    c, s = table[pos, :rot // 2].double()[:, None], table[pos, rot // 2:].double()[:, None] * (-1 if back else 1)
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([r, x[..., rot:]], -1)


# ------------------------------------------------------------- norms of heads

def heads64(x, w, d, eps, table, pos, inter):
    h = x.double().unflatten(1, (-1, d))
    rstd = 1.0 / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    n = h * rstd * (1.0 if w is None else w.double())
    return h, rstd, n, turn64(n, table, pos, inter).flatten(1)


def head_bound(n, table, inter, d):
    """Roundings of a norm of d values (the sum of squares d / 2 + 3 of them, of which rstd has half; rstd, weight and
    products 5) and of the rotation (4) relative to the two numbers of a pair."""
    big = n.abs()
    if table is not None:
        rot = table.shape[1]
        one = torch.ones_like(table[:1])
        one[:, rot // 2:] = -1                                  # |a| + |b| by a turn with c = 1, s = -1 of magnitudes
        z = torch.zeros(n.shape[0], dtype=torch.int64, device=n.device)
        pair = turn64(big, one, z, inter)
        lower = turn64(big, torch.ones_like(one), z, inter)
        big = torch.maximum(big, torch.maximum(pair.abs(), lower.abs()))
    return (((d / 2 + 3) / 2 + 9) * U * big).flatten(1)


SHAPES = [(1, 32, 8, 128, 128, False), (7, 3, 1, 64, 64, True), (5, 4, 2, 96, 24, False), (300, 5, 5, 80, 80, False), (3, 2, 2, 256, 256, False),
          (2, 1, 1, 8, 6, False), (9, 2, 1, 40, 0, False), (4, 7, 1, 72, 18, True), (2600, 8, 2, 128, 64, False), (3, 3, 2, 248, 128, True),
          (11, 1, 1, 16, 16, False), (2, 6, 2, 160, 32, True)]


@pytest.mark.parametrize("n,hq,hk,d,rot,inter", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_headnorm_and_gradient(n, hq, hk, d, rot, inter, dtype):
    eps = 1e-5
    r = esb.rotation(rot, 5000, 500000.0, interleaved=inter) if rot else None
    pos = ints(0, 5000, (n,), 3)
    table = r.table if r else None
    qkv = rand((n, (hq + 2 * hk) * d), 1, dtype, 2.0)
    q, k = qkv[:, :hq * d], qkv[:, hq * d:(hq + hk) * d]
    wq, wk = 1 + rand((d,), 2, std=0.1), 1 + rand((d,), 3, std=0.1)
    out = esb.esb_headnorm(q, k, d, wq, wk, eps, rotation=r, positions=pos, want_rstd=True)
    gq, gk = rand((n, hq * d), 4, dtype), rand((n, hk * d), 5, dtype)
    b = esb.esb_headnorm_backward(gq, gk, q, k, d, wq, wk, out.q_rstd, out.k_rstd, rotation=r, positions=pos)
    for x, w, y, rs, g, dx, dw in ((q, wq, out.q, out.q_rstd, gq, b.dq, b.dq_weight), (k, wk, out.k, out.k_rstd, gk, b.dk, b.dk_weight)):
        h, rstd, m, y64 = heads64(x, w, d, eps, table, pos, inter)
        close(y, y64, head_bound(m, table, inter, d), dtype)
        close(rs, rstd[..., 0], ((d / 2 + 3) / 2 + 4) * U * rstd[..., 0], FL)
        dy = turn64(g.double().unflatten(1, (-1, d)), table, pos, inter, back=True)
        e, hn = dy * w.double(), h * rstd
        dot = (e * hn).mean(-1, keepdim=True)
        # e: rotation and weight (5 roundings of the pair's size), n: 40 of rstd at most; the dot product's d / 2 + 12 of the
        # sum of magnitudes; each is counted by the largest number of the pair or head that it comes from
        big = (g.double().unflatten(1, (-1, d)).abs().amax(-1, keepdim=True) * 2 * w.double().abs().max())
        bound = rstd * U * ((12 + d / 4) * big + hn.abs() * (big * hn.abs()).mean(-1, keepdim=True) * (60 + d))
        close(dx, (rstd * (e - hn * dot)).flatten(1), bound.flatten(1), dtype)
        terms = dy * hn
        # every term has some 10 + d / 4 roundings (rstd's), their sum at most as many as a lane adds and joins
        size = (big / w.double().abs().max() * hn.abs()).sum((0, 1))
        close(dw, terms.sum((0, 1)), size * U * (12 + d / 4 + n * hq / 200 + 30), FL)


def test_headnorm_gradient_against_differences():
    # the formula's own check: the 64-bit gradient above and differences of the 64-bit forward pass
    d, n = 16, 3
    r = esb.rotation(8, 50)
    pos = ints(0, 50, (n,), 1)
    x, w, g = rand((n, 2 * d), 2).double(), 1 + rand((d,), 3, std=0.2).double(), rand((n, 2 * d), 4).double()

    def f(x, w):
        return (heads64(x, w, d, 1e-6, r.table, pos, False)[3] * g).sum()
    out = esb.esb_headnorm(x.float(), None, d, w.float(), None, rotation=r, positions=pos, want_rstd=True)
    b = esb.esb_headnorm_backward(g.float(), None, x.float(), None, d, w.float(), None, out.q_rstd, None, rotation=r, positions=pos)
    h = 1e-5
    for i, j in [(0, 0), (1, 5), (2, 31), (0, 17)]:
        e = torch.zeros_like(x)
        e[i, j] = h
        # a central difference is off by h^2 / 6 of a third derivative (below 100 here) and 1e-16 / h of rounding
        assert abs(float((f(x + e, w) - f(x - e, w)) / (2 * h)) - float(b.dq[i, j])) < 1e-5
    for j in (0, 3, 15):
        e = torch.zeros_like(w)
        e[j] = h
        assert abs(float((f(x, w + e) - f(x, w - e)) / (2 * h)) - float(b.dq_weight[j])) < 1e-5


@pytest.mark.parametrize("dtype", TYPES)
def test_headnorm_in_place_strides_and_parts(dtype):
    n, d, hq, hk = 21, 64, 5, 3
    r = esb.rotation(64, 100)
    pos = ints(0, 100, (n,), 1)
    wide = rand((n, (hq + hk) * d + 9), 2, dtype)
    q, k = wide[:, 1:1 + hq * d], wide[:, 3 + hq * d:3 + (hq + hk) * d]      # rows that start anywhere
    w = 1 + rand((d,), 5, dtype, 0.1)
    want = esb.esb_headnorm(q.contiguous(), k.contiguous(), d, w, None, rotation=r, positions=pos)
    got = esb.esb_headnorm(q, k, d, w, None, rotation=r, positions=pos)
    assert torch.equal(got.q, want.q) and torch.equal(got.k, want.k) and got.q_rstd is None
    only = esb.esb_headnorm(None, k, d, None, None, rotation=r, positions=pos, want_rstd=True)
    assert only.q is None and torch.equal(only.k, want.k) and only.k_rstd.shape == (n, hk)
    before = wide.clone()
    esb.esb_headnorm(q, k, d, w, None, rotation=r, positions=pos, qy=q, ky=k)
    assert torch.equal(q, want.q) and torch.equal(k, want.k)
    assert torch.equal(wide[:, :1], before[:, :1]) and torch.equal(wide[:, -6:], before[:, -6:])
    # no tokens: gradients of the weights are zeros
    none = torch.empty((0, d), dtype=dtype, device="cuda")
    out = esb.esb_headnorm(none, none, d, w, w, want_rstd=True)
    b = esb.esb_headnorm_backward(none, none, none, none, d, w, w, out.q_rstd, out.k_rstd)
    assert out.q.shape == (0, d) and (b.dq_weight == 0).all() and (b.dk_weight == 0).all()


def test_headnorm_special_values_and_far_positions():
    n, d = 6, 128
    r = esb.rotation(d, 4)
    pos = torch.tensor([0, 3, 4, -1, 1 << 40, 2], device="cuda")
    x = rand((n, d), 1)
    x[5, 7] = float("inf")
    y = esb.esb_headnorm(x, None, d, rotation=r, positions=pos).q
    assert torch.isfinite(y[:2]).all() and torch.isnan(y[2:5]).all() and torch.isnan(y[5]).any()
    z = esb.esb_headnorm(torch.zeros((2, d), device="cuda"), None, d, eps=1e-6).q
    assert (z == 0).all()
    # position 0 turns by nothing
    assert torch.equal(esb.esb_headnorm(x[:1], None, d, rotation=r, positions=pos[:1]).q, esb.esb_headnorm(x[:1], None, d).q)


def test_headnorm_repeats_on_another_stream_and_in_a_graph():
    n, d = 700, 128
    r = esb.rotation(d, 1000)
    pos = torch.arange(n, device="cuda")
    q, g, w = rand((n, 4 * d), 1, BF), rand((n, 4 * d), 2, BF), 1 + rand((d,), 3, std=0.1)

    def step(stream=None, q=q):
        out = esb.esb_headnorm(q, q[:, :d], d, w, w, rotation=r, positions=pos, want_rstd=True, stream=stream)
        return out, esb.esb_headnorm_backward(g, g[:, :d], q, q[:, :d], d, w, w, out.q_rstd, out.k_rstd, rotation=r, positions=pos, stream=stream)
    want = step()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = step(st)
    st.synchronize()
    q2 = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(q=q2)
    graph.replay()
    torch.cuda.synchronize()
    for other in (got, held, step()):
        for x, y in zip(want, other):
            for a, b in zip(x, y):
                assert torch.equal(a, b)
    q2.mul_(2.0)
    graph.replay()
    assert torch.equal(held[0].q, step(q=q2)[0].q)


# --------------------------------------------------------------------- append

def rows_of(codes, scales, slots, page):
    return codes[slots // page, :, slots % page], scales[slots // page, :, slots % page]


APPENDS = [(37, 8, 128, 128, False, 16), (1, 1, 64, 64, False, 32), (130, 3, 96, 24, False, 48), (9, 2, 80, 80, True, 64), (20, 5, 256, 256, False, 16),
           (17, 2, 8, 6, False, 16), (50, 1, 72, 0, False, 16), (33, 4, 40, 40, False, 32), (12, 2, 248, 128, True, 16), (700, 4, 128, 64, False, 128)]


@pytest.mark.parametrize("n,heads,d,rot,inter,page", APPENDS)
@pytest.mark.parametrize("dtype", TYPES)
def test_append_is_the_projection_of_rotated_rows(n, heads, d, rot, inter, page, dtype):
    pages = -(-n // page) + 2
    r = esb.rotation(rot, 3000, interleaved=inter) if rot else None
    pos = ints(0, 3000, (n,), 1)
    qkv = rand((n, 3 * heads * d + 5), 2, dtype)
    k, v = qkv[:, heads * d:2 * heads * d], qkv[:, 2 * heads * d:3 * heads * d]
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n]
    left = slots.clone()
    if n > 3:
        left[1], left[3] = -1, pages * page                      # left out
    on = (left >= 0) & (left < pages * page)
    for i, (kk, vk, rule, rounding) in enumerate([(2, 1, 0, 0), (0, 3, 0, 1), (2, 2, 1, 0)]):
        c = esb.kv_cache(pages, heads, page, d, esb.Fmt(4, kk), esb.Fmt(4, vk))
        for t in (c.k_codes, c.v_codes):
            t.fill_(77)
        for t in (c.k_scales, c.v_scales):
            t.fill_(-5.0)
        kq, vq = (torch.full((n, heads * d), 9.0, dtype=[FL, BF, HF][i], device="cuda") for _ in range(2))
        esb.esb_cache_append(c, k, v, left, rotation=r, positions=pos if r else None, rule=rule, rounding=rounding, kq=kq, vq=vq)
        for x, codes, scales, f, q in ((k, c.k_codes, c.k_scales, c.k_fmt, kq), (v, c.v_codes, c.v_scales, c.v_fmt, vq)):
            h = x.double().unflatten(1, (heads, d))
            if x is k:
                h = turn64(h, r.table if r else None, pos, inter)
            want, xq = esb.esb_project_groups(h.float().flatten(0, 1), f, 0, rule=rule, rounding=rounding,
                                              xq=torch.empty((n * heads, d), dtype=q.dtype, device="cuda"))
            gc, gs = rows_of(codes, scales, left[on], page)
            ws = want.scales.unflatten(0, (n, heads))[on][..., 0]
            if rule == 0:
                assert torch.equal(gs, ws)
                assert torch.equal(gc, want.codes.unflatten(0, (n, heads))[on])
                assert torch.equal(q[on], xq.unflatten(0, (n, heads))[on].flatten(1))
            else:
                # the spread's sums go in another order: d / 2 roundings of it in each
                assert ((gs - ws).abs() <= (d / 2 + 8) * 2 * U * ws).all()
                again = o.unpack(gc.flatten(0, 1).cpu().numpy().view("uint32"), d, 4)
                rows = h.float()[on].flatten(0, 1).cpu().numpy()
                for j in range(0, rows.shape[0], 7):
                    assert (again[j] == o.project_codes(rows[j], float(gs.flatten()[j]), 4, f.k, True, rounding)).all()
            assert (q[~on] == 9).all()
            rest = torch.ones(pages * page, dtype=torch.bool, device="cuda")
            rest[left[on]] = False
            at = torch.nonzero(rest)[:, 0]
            oc, os = rows_of(codes, scales, at, page)
            assert (oc == 77).all() and (os == -5).all()


def test_append_special_values_and_page_strides():
    # a cache whose pages lie between others' (layers of one allocation); zeros, NaN and infinities; a far position
    pages, heads, page, d = 3, 2, 16, 64
    codes = torch.full((pages, 2, 3, heads, page, 8), 5, dtype=torch.int32, device="cuda")
    scales = torch.full((pages, 2, 3, heads, page), 5.0, device="cuda")
    c = esb.KvCache(codes[:, 0, 1], scales[:, 0, 1], codes[:, 1, 1], scales[:, 1, 1], d, esb.Fmt(4, 2), esb.Fmt(4, 2))
    k, v = rand((5, heads * d), 1), rand((5, heads * d), 2)
    k[0] = 0
    v[1, 3] = float("nan")
    v[2, 70] = -float("inf")
    r = esb.rotation(64, 10)
    pos = torch.tensor([1, 2, 3, 10, 4], device="cuda")
    slots = torch.tensor([47, 0, 17, 18, 31], device="cuda")
    esb.esb_cache_append(c, k, v, slots, rotation=r, positions=pos)
    ks, vs = (t[slots // page, :, slots % page] for t in (c.k_scales, c.v_scales))
    assert (ks[0] == 0).all() and torch.isnan(ks[3]).all() and torch.isnan(vs[1, 0]) and torch.isinf(vs[2, 1]) and torch.isfinite(vs[0]).all()
    zero = esb.esb_zero_code(esb.Fmt(4, 2)) * 0x11111111
    zero = zero - (1 << 32) if zero >= 1 << 31 else zero
    assert (c.k_codes[2, :, 15] == zero).all() and (c.v_codes[0, 0, 0] == zero).all() and (c.v_codes[1, 1, 1] == zero).all()
    touched = torch.zeros_like(codes, dtype=torch.bool)
    touched[slots // page, :, 1, :, slots % page] = True
    assert (codes[~touched] == 5).all()
    # nothing to do
    esb.esb_cache_append(c, k[:0], v[:0], slots[:0], rotation=r, positions=pos[:0])
    empty = esb.kv_cache(0, heads, page, d)
    esb.esb_cache_append(empty, k, v, slots)


# ------------------------------------------------------------------ attention

def make_cache(pages, heads, page, d, kk, vk, seed, spread=0.3):
    c = esb.kv_cache(pages, heads, page, d, esb.Fmt(4, kk), esb.Fmt(4, vk))
    n = pages * page
    for at in range(0, n, 1 << 16):
        m = min(1 << 16, n - at)
        size = torch.exp(spread * rand((m, 1), seed + 2))
        esb.esb_cache_append(c, rand((m, heads * d), seed) * size, rand((m, heads * d), seed + 1) * size, torch.arange(at, at + m, device="cuda"))
    return c


def cached64(c, which, pages):
    """Values (heads, places, d) of the pages of a list."""
    codes, scales, f = (c.k_codes, c.k_scales, c.k_fmt) if which == "k" else (c.v_codes, c.v_scales, c.v_fmt)
    w, s = codes[pages].transpose(0, 1).flatten(1, 2), scales[pages].transpose(0, 1).flatten(1, 2)
    table = torch.tensor([o.decode(x, 4, f.k) for x in range(16)], dtype=F64, device="cuda")
    v = table[torch.stack([(w >> (4 * i)) & 15 for i in range(8)], -1).flatten(-2)[..., :c.head_dim].long()]
    return v * s.double()[..., None], s.double()


def check_attention(q, c, lens, pages, out, lse, starts=None, scale=None, rotation=None, window=0, every=1):
    """Every sequence's queries (or every so many rows of them) against 64 bits, with the bound of the roundings."""
    d, heads, page = c.head_dim, c.k_codes.shape[1], c.k_codes.shape[2]
    group = q.shape[1] // d // heads
    scale = d ** -0.5 if scale is None else scale
    coarse = 2.0 ** -11 if q.dtype == BF else 2.0 ** -21       # roundings of queries and of weights to fp16 (or two of them)
    top = max(o.decode(x, 4, c.v_fmt.k) for x in range(16))
    for i, n in enumerate(lens.tolist()):
        r0, r1 = (i, i + 1) if starts is None else (int(starts[i]), int(starts[i + 1]))
        m = r1 - r0
        if m <= 0:
            continue
        pick = torch.arange(0, m, every, device="cuda")
        pos = n - m + pick
        x = q[r0:r1][pick].double().unflatten(1, (heads * group, d))
        if rotation is not None:
            x = turn64(x, rotation.table, pos.clamp_min(0), rotation.interleaved)
        held = min(max(n, 0), pages.shape[1] * page)
        at = pages[i, :-(-held // page)].long()
        there = ((at >= 0) & (at < c.k_codes.shape[0])).repeat_interleave(page)[:held]
        at = at.clamp(0, c.k_codes.shape[0] - 1)
        (k, _), (v, vs) = cached64(c, "k", at), cached64(c, "v", at)
        p = torch.arange(held, device="cuda")
        seen = (p[None] <= pos[:, None]) & there[None]
        if window:
            seen &= p[None] > pos[:, None] - window
        for h in range(heads):
            kh, vh, vsh = k[h, :held], v[h, :held], vs[h, :held]
            # what no query sees may be anything
            any_seen = seen.any(0)
            kh = torch.where(any_seen[:, None], kh, torch.zeros_like(kh))
            vh = torch.where(any_seen[:, None], vh, torch.zeros_like(vh))
            vsh = torch.where(any_seen, vsh, torch.zeros_like(vsh))
            for j in range(h * group, (h + 1) * group):
                s = (x[:, j] @ kh.t() * scale).masked_fill(~seen, -math.inf)
                has = seen.any(1)
                mx = torch.where(has, s.amax(1) if held else torch.zeros(len(pick), device="cuda", dtype=F64), torch.zeros(len(pick), device="cuda", dtype=F64))
                e = torch.exp(s - mx[:, None])
                l = e.sum(1, keepdim=True)
                pr = torch.where(l > 0, e / l, torch.zeros_like(e))
                want = pr @ vh
                # a score: its query's rounding, d sums and 8 products and sums of fp32; the exponent's own
                size = x[:, j].abs() @ kh.abs().t() * abs(scale)
                ds = size * (coarse + (d + 12) * U) + 16 * U * torch.where(seen, (s - mx[:, None]).abs() + mx.abs()[:, None], torch.zeros_like(s))
                eta = torch.expm1(ds) + coarse + 2.0 ** -20
                # weights are fp16 with steps of 2^-24 below 2^-14, the largest of them is above 1/2
                u = torch.where(seen, e * vsh.clamp_min(2.0 ** -100), torch.zeros_like(e))
                least = u.amax(1, keepdim=True) * 2.0 ** -24 * top * seen.sum(1, keepdim=True) / l.clamp_min(1e-300) if held else 0.0
                spread = pr * eta
                sums = (held + 64) * U
                bound = spread @ vh.abs() + want.abs() * (spread.sum(1, keepdim=True) + sums) + (pr @ vh.abs()) * sums + least
                got = out[r0:r1][pick][:, j * d:(j + 1) * d]
                close(got[has], want[has], bound[has], got.dtype)
                assert (got[~has] == 0).all()
                if lse is not None:
                    gl = lse[r0:r1][pick][:, j].double()
                    assert (gl[~has] == -math.inf).all()
                    wl = mx + torch.log(l[:, 0])
                    # the logarithm of a sum whose terms are off by eta each
                    tol = torch.log1p(spread.sum(1)) * 1.01 + sums + 8 * U * (wl.abs() + mx.abs()) + 2.0 ** -20
                    assert ((gl - wl).abs()[has] <= tol[has]).all(), float(((gl - wl).abs() / tol)[has].max())


def tables(lens, page, pages, seed):
    """Page tables of distinct pages out of `pages`, every sequence's on random ones."""
    most = max(1, max(-(-max(n, 0) // page) for n in lens))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    t = torch.full((len(lens), most), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(lens):
        m = -(-max(n, 0) // page)
        t[i, :m] = order[at:at + m]
        at += m
    return t


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


DECODE = [  # lens, heads, group, d, page, kk, vk, rot, inter, window
    ([1], 1, 1, 64, 16, 2, 2, 0, False, 0),
    ([1, 2, 15, 16, 17, 63, 64, 65, 100, 0, 1000], 2, 4, 128, 16, 2, 2, 128, False, 0),
    ([3000, 5, 0, 777], 8, 4, 128, 64, 2, 1, 128, False, 0),
    ([129, 513, 300], 3, 7, 96, 48, 0, 3, 24, True, 0),
    ([400, 1, 250], 2, 8, 80, 32, 1, 0, 80, False, 0),
    ([640, 33], 4, 1, 256, 16, 3, 2, 256, False, 0),
    ([900, 64, 65], 1, 16, 128, 128, 2, 2, 64, True, 0),
    ([500, 20], 2, 12, 64, 16, 2, 2, 64, False, 0),
    ([700, 90], 2, 24, 128, 32, 2, 2, 0, False, 0),
    ([300, 31], 1, 40, 64, 16, 2, 2, 64, False, 17),
    ([1000, 5, 99, 100, 101], 2, 4, 128, 16, 2, 2, 128, False, 100),
    ([222, 48], 2, 5, 256, 16, 2, 2, 64, False, 1),
    ([222, 48], 2, 2, 8, 16, 2, 2, 6, False, 40),
    ([100, 7], 1, 9, 248, 32, 1, 2, 0, False, 0),
    ([40000], 2, 4, 128, 64, 2, 2, 128, False, 0),
]


@pytest.mark.parametrize("case", range(len(DECODE)))
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_single_tokens(case, dtype):
    lens, heads, group, d, page, kk, vk, rot, inter, window = DECODE[case]
    pages = sum(-(-n // page) for n in lens) + 3
    c = make_cache(pages, heads, page, d, kk, vk, 5)
    t = tables(lens, page, pages, 7)
    r = esb.rotation(rot, max(lens) + 1, interleaved=inter) if rot else None
    q = rand((len(lens), heads * group * d), 8, dtype)
    out, lse = esb.esb_cache_attention(q, c, i32(lens), t, rotation=r, window=window, want_lse=True)
    check_attention(q, c, i32(lens), t, out, lse, rotation=r, window=window)
    again, none = esb.esb_cache_attention(q, c, i32(lens), t, rotation=r, window=window)
    assert torch.equal(out, again) and none is None


SEVERAL = [  # (queries, places) of each sequence, heads, group, d, page, kk, vk, rot, window
    ([(4, 100), (1, 50), (0, 30), (3, 3), (2, 1), (5, 0)], 2, 4, 128, 16, 2, 2, 128, 0),
    ([(17, 400), (33, 33), (1, 300)], 1, 3, 96, 48, 0, 1, 32, 0),
    ([(130, 1000), (64, 64)], 2, 4, 128, 32, 2, 2, 128, 0),
    ([(130, 300), (7, 500)], 1, 8, 256, 16, 2, 3, 256, 0),
    ([(200, 700), (9, 90)], 2, 5, 64, 64, 1, 2, 64, 33),
    ([(2, 3000), (2, 2000), (2, 10)], 4, 8, 128, 64, 2, 2, 128, 1000),
    ([(1200, 1200)], 1, 8, 64, 16, 2, 2, 64, 0),
    ([(1, 77)] * 150 + [(40, 500)] + [(0, 0)] * 200 + [(3, 64)], 1, 2, 64, 16, 2, 2, 64, 0),
]


@pytest.mark.parametrize("case", range(len(SEVERAL)))
@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_several_tokens(case, dtype):
    seqs, heads, group, d, page, kk, vk, rot, window = SEVERAL[case]
    lens = [n for _, n in seqs]
    pages = sum(-(-n // page) for n in lens) + 3
    c = make_cache(pages, heads, page, d, kk, vk, 5)
    t = tables(lens, page, pages, 7)
    starts = [2]                                                  # rows before the first and behind the last sequence
    for m, _ in seqs:
        starts.append(starts[-1] + m)
    r = esb.rotation(rot, max(lens) + 1)
    q = rand((starts[-1] + 3, heads * group * d), 8, dtype)
    out = torch.full_like(q, 7.0)
    _, lse = esb.esb_cache_attention(q, c, i32(lens), t, starts=i32(starts), rotation=r, window=window, out=out, want_lse=True)
    check_attention(q, c, i32(lens), t, out, lse, starts=i32(starts), rotation=r, window=window, every=1 if max(lens) < 600 else 7)
    assert (out[:2] == 7).all() and (out[starts[-1]:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_does_not_see_what_it_must_not(dtype):
    # NaN scales behind a sequence's end, before a window and on other pages; pages that are not there; a length past
    # the table
    heads, group, d, page = 2, 4, 128, 16
    lens = [37, 100, 64, 1000]
    c = make_cache(40, heads, page, d, 2, 2, 3)
    t = torch.full((4, 10), 39, dtype=torch.int32, device="cuda")
    t[0, :3], t[1, :7], t[2, :4], t[3, :10] = i32([5, 1, 8]), i32([2, -1, 3, 4, 99, 6, 7]), i32([-1, -1, 40, -7]), torch.arange(10, 20, device="cuda")
    for s in (c.k_scales, c.v_scales):
        s[39], s[8, :, 5:], s[7, :, 4:] = float("nan"), float("inf"), float("nan")
        s[0], s[20:39] = float("nan"), float("nan")
    q = rand((4, heads * group * d), 8, dtype)
    for window in (0, 20):
        if window:
            for s in (c.k_scales, c.v_scales):
                s[5, :, :], s[1, :, 0] = float("nan"), float("nan")
        out, lse = esb.esb_cache_attention(q, c, i32(lens), t, window=window, want_lse=True)
        check_attention(q, c, i32(lens), t, out, lse, window=window)
        assert (out[2] == 0).all() and (lse[2] == -math.inf).all()
        assert torch.isfinite(out).all()
        if window:
            assert (out[3] == 0).all()                             # its last 20 places are past the table
    # and what it sees makes it NaN
    c.v_scales[12, 1, 3] = float("nan")
    out, lse = esb.esb_cache_attention(q, c, i32(lens), t, want_lse=True)
    assert torch.isnan(out[3, group * d:]).all() and torch.isfinite(out[3, :group * d]).all() and torch.isfinite(lse[3]).all()
    c.k_scales[12, 0, 3] = float("nan")
    out, lse = esb.esb_cache_attention(q, c, i32(lens), t, want_lse=True)
    assert torch.isnan(out[3]).all() and torch.isnan(lse[3, :group]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_scales_of_any_size(dtype):
    # values' scales over sixty orders of two, a few places far ahead of the others, queries near the type's ends
    heads, group, d, page, n = 1, 4, 64, 16, 300
    c = make_cache(19, heads, page, d, 2, 2, 3)
    t = torch.arange(19, dtype=torch.int32, device="cuda")[None]
    c.v_scales.mul_(torch.exp2(ints(-40, 20, c.v_scales.shape, 5).float()))
    q = rand((1, heads * group * d), 8, dtype)
    for scale in (None, 3.0, 0.0, -1.0, 1e-3):
        out, lse = esb.esb_cache_attention(q, c, i32([n]), t, scale=scale, out=torch.empty_like(q, dtype=FL), want_lse=True)
        check_attention(q, c, i32([n]), t, out, lse, scale=scale)
    big = (q.float() * torch.finfo(dtype).max / 8).to(dtype) if dtype != FL else q * 1e30
    small = (q.float() * 2.0 ** -20).to(dtype)
    near = (q.float() * (torch.finfo(dtype).max / 8)).to(dtype)
    for x, scale in ((big, 1.0 / float(big.float().abs().max())), (small, 1.0), (near, 1.0 / float(near.float().abs().max()))):
        out, lse = esb.esb_cache_attention(x, c, i32([n]), t, scale=scale, out=torch.empty_like(q, dtype=FL), want_lse=True)
        if torch.isfinite(x).all():
            check_attention(x, c, i32([n]), t, out, lse, scale=scale)
        else:                                                      # bf16: products past fp32's range in every head
            assert dtype == BF and torch.isinf(x.unflatten(1, (-1, d))).any(-1).all() and torch.isnan(out).all() and torch.isnan(lse).all()
    c.v_scales.zero_()
    out, lse = esb.esb_cache_attention(q, c, i32([n]), t, want_lse=True)
    assert (out == 0).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_strides_and_page_strides(dtype):
    heads, group, d, page = 2, 3, 96, 16
    lens = [150, 31, 70]
    pages = 20
    c = make_cache(pages, heads, page, d, 2, 1, 3)
    codes = torch.zeros((pages, 2, 3, heads, page, 12), dtype=torch.int32, device="cuda")
    scales = torch.full((pages, 2, 3, heads, page), float("nan"), device="cuda")
    codes[:, 0, 1], codes[:, 1, 1], scales[:, 0, 1], scales[:, 1, 1] = c.k_codes, c.v_codes, c.k_scales, c.v_scales
    c2 = esb.KvCache(codes[:, 0, 1], scales[:, 0, 1], codes[:, 1, 1], scales[:, 1, 1], d, c.k_fmt, c.v_fmt)
    t = tables(lens, page, pages, 1)
    wide_t = torch.full((3, t.shape[1] + 5), 3, dtype=torch.int32, device="cuda")
    wide_t[:, 2:2 + t.shape[1]] = t
    r = esb.rotation(d, 200)
    wide = rand((3, heads * group * d + 40), 8, dtype)
    out = torch.full_like(wide, 4.0)
    q = wide[:, 3:3 + heads * group * d]
    want, wl = esb.esb_cache_attention(q.contiguous(), c, i32(lens), t, rotation=r, want_lse=True)
    got, gl = esb.esb_cache_attention(q, c2, i32(lens), wide_t[:, 2:2 + t.shape[1]], rotation=r, out=out[:, 5:5 + heads * group * d], want_lse=True)
    assert torch.equal(got, want) and torch.equal(gl, wl)
    assert (out[:, :5] == 4).all() and (out[:, 5 + heads * group * d:] == 4).all()


def test_attention_offsets_past_32_bits():
    # pages more than 2^32 words apart
    heads, page, d = 2, 16, 64
    c = make_cache(3, heads, page, d, 2, 2, 3)
    gap = (1 << 31) + 64
    store = torch.empty(2 * gap + heads * page * 8, dtype=torch.int32, device="cuda")
    kc = torch.as_strided(store, (3, heads, page, 8), (gap, page * 8, 8, 1))
    kc.copy_(c.k_codes)
    vc = torch.as_strided(store, (3, heads, page, 8), (gap, page * 8, 8, 1), storage_offset=0)
    c2 = esb.KvCache(kc, c.k_scales, vc, c.v_scales, d, c.k_fmt, c.v_fmt)
    t, lens = i32([[2, 0, 1]]), i32([45])
    q = rand((1, heads * 2 * d), 1)
    want, _ = esb.esb_cache_attention(q, c._replace(v_codes=c.k_codes), lens, t)
    assert torch.equal(esb.esb_cache_attention(q, c2, lens, t)[0], want)
    x = rand((1, heads * d), 2)
    for y in (c2, c):
        esb.esb_cache_append(y._replace(v_codes=y.v_codes), x, x, torch.tensor([2 * page + 5], device="cuda"))
    assert torch.equal(kc[2, :, 5], c.k_codes[2, :, 5])


@pytest.mark.parametrize("seqs", [128, 129, 1500, 17000])
def test_attention_of_many_sequences(seqs):
    # more sequences than threads that look for a block's part of them, some without queries, some with many
    g = torch.Generator(device="cuda")
    g.manual_seed(seqs)
    c = make_cache(50, 1, 16, 64, 2, 2, 3)
    lens = torch.randint(0, 60, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randint(0, 50, (seqs, 4), generator=g, device="cuda", dtype=torch.int32)
    q = rand((seqs, 64), 8, BF)
    out, lse = esb.esb_cache_attention(q, c, lens, t, want_lse=True)
    pick = torch.cat([torch.arange(0, seqs, max(1, seqs // 40), device="cuda"), torch.tensor([seqs - 1], device="cuda")])
    check_attention(q[pick], c, lens[pick], t[pick], out[pick], lse[pick])
    # the same as several queries of some
    counts = torch.randint(0, 3, (seqs,), generator=g, device="cuda")
    counts[seqs // 2], counts[seqs // 3] = 300, 90
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    q = rand((int(starts[-1]), 64), 9, BF)
    out, lse = esb.esb_cache_attention(q, c, lens, t, starts=starts, want_lse=True)
    for i in pick.tolist() + [seqs // 2, seqs // 3]:
        a, b = int(starts[i]), int(starts[i + 1])
        check_attention(q[a:b], c, lens[i:i + 1], t[i:i + 1], out[a:b], lse[a:b], starts=i32([0, b - a]))


def test_rows_past_32_bits():
    # tokens' rows more than 2^31 values apart, into and out of each operator
    d, n, ld = 64, 3, (1 << 31) + 8
    store = torch.empty((n - 1) * ld + 2 * d, dtype=BF, device="cuda")
    far = torch.as_strided(store, (n, 2 * d), (ld, 1))
    x = rand((n, 2 * d), 1, BF)
    far.copy_(x)
    r, pos = esb.rotation(d, 10), ints(0, 10, (n,), 2)
    want = esb.esb_headnorm(x, None, d, rotation=r, positions=pos, want_rstd=True)
    assert torch.equal(esb.esb_headnorm(far, None, d, rotation=r, positions=pos).q, want.q)
    g = rand((n, 2 * d), 3, BF)
    dw = 1 + rand((d,), 4, std=0.1)
    b = esb.esb_headnorm_backward(g, None, x, None, d, dw, None, want.q_rstd, None, rotation=r, positions=pos)
    bf = esb.esb_headnorm_backward(g, None, far, None, d, dw, None, want.q_rstd, None, rotation=r, positions=pos)
    assert torch.equal(b.dq, bf.dq) and torch.equal(b.dq_weight, bf.dq_weight)
    slots = torch.tensor([3, 20, 4], device="cuda")
    near, wide = esb.kv_cache(2, 2, 16, d), esb.kv_cache(2, 2, 16, d)
    esb.esb_cache_append(near, x, x, slots, rotation=r, positions=pos)
    esb.esb_cache_append(wide, far, far, slots, rotation=r, positions=pos)
    assert torch.equal(near.k_codes, wide.k_codes) and torch.equal(near.v_codes, wide.v_codes) and torch.equal(near.k_scales, wide.k_scales)
    t, lens = i32([[0, 1]] * n), i32([32, 5, 21])
    a, _ = esb.esb_cache_attention(x, near, lens, t)
    assert torch.equal(esb.esb_cache_attention(far, near, lens, t, out=far)[0], a)   # the output on the queries' own rows


def test_attention_nothing_to_do_and_refusals():
    c = esb.kv_cache(2, 1, 16, 64)
    q = rand((2, 64), 1)
    t = i32([[0], [1]])
    out, lse = esb.esb_cache_attention(q[:0], c, i32([]), t[:0], want_lse=True)
    assert out.shape == (0, 64) and lse.shape == (0, 1)
    out, _ = esb.esb_cache_attention(q, c, i32([0, -5]), t)
    assert (out == 0).all()
    out, _ = esb.esb_cache_attention(q, c, i32([4, 4]), torch.empty((2, 0), dtype=torch.int32, device="cuda"))
    assert (out == 0).all()
    out, _ = esb.esb_cache_attention(q, esb.kv_cache(0, 1, 16, 64), i32([4, 4]), t)
    assert (out == 0).all()
    for call in (lambda: esb.esb_cache_attention(q, c, i32([1]), t), lambda: esb.esb_cache_attention(q, c, i32([1, 1, 1]), i32([[0]] * 3)),
                 lambda: esb.esb_cache_attention(q[:, :60], c, i32([1, 1]), t), lambda: esb.esb_cache_attention(q, c, i32([1, 1]), t, out=q[:1]),
                 lambda: esb.esb_cache_attention(q, c, i32([1, 1]), t.long()), lambda: esb.esb_cache_append(c, q, q[:1], torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: esb.esb_cache_append(c, q, q, i32([0, 1])), lambda: esb.esb_headnorm(q, None, 60)):
        with pytest.raises((ValueError, esb.EsbError)):
            call()


def test_attention_calls_share_a_workspace_one_after_the_other():
    # a call's parts are joined before the next call writes its own, whatever the shapes; two streams have a workspace each
    c, small = make_cache(300, 4, 64, 128, 2, 1, 3), make_cache(40, 2, 16, 64, 0, 2, 4)
    t, ts = tables([9000, 5000, 100], 64, 300, 1), tables([300, 20], 16, 40, 2)
    n, ns, starts = i32([9000, 5000, 100]), i32([300, 20]), i32([0, 12, 20])
    q, qs, qf = rand((3, 16 * 128), 1, BF), rand((20, 6 * 64), 2, HF), rand((3, 8 * 128), 3)
    nb = 1 << 26
    calls = [lambda w, s: esb.esb_cache_attention(q, c, n, t, want_lse=True, workspace=w, stream=s),
             lambda w, s: esb.esb_cache_attention(qs, small, ns, ts, starts=starts, want_lse=True, workspace=w, stream=s),
             lambda w, s: esb.esb_cache_attention(qf, c, n, t, want_lse=True, window=3000, workspace=w, stream=s)]
    want = [f(None, None) for f in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.full((nb,), 255, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    got = [[f(w, s) for _ in range(8) for f in calls] for w, s in zip(spaces, streams)]
    torch.cuda.synchronize()
    for outs in got:
        for i, (o1, l1) in enumerate(outs):
            assert torch.equal(o1, want[i % 3][0]) and torch.equal(l1, want[i % 3][1]), i
    with pytest.raises(esb.EsbError):
        calls[0](spaces[0][:1000], None)


def test_attention_repeats_on_another_stream_and_in_a_graph():
    heads, group, d, page = 8, 4, 128, 64
    lens = [5000, 300, 12000, 64]
    pages = sum(-(-n // page) for n in lens)
    c = make_cache(pages, heads, page, d, 2, 2, 3)
    t = tables(lens, page, pages, 1)
    r = esb.rotation(d, 12001)
    q = rand((4, heads * group * d), 8, BF)
    want, wl = esb.esb_cache_attention(q, c, i32(lens), t, rotation=r, want_lse=True)
    check_attention(q, c, i32(lens), t, want, wl, rotation=r)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    n = i32(lens)
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        got, gl = esb.esb_cache_attention(q, c, n, t, rotation=r, want_lse=True, stream=st)
        st.synchronize()
        assert torch.equal(got, want) and torch.equal(gl, wl)
    q2, n2 = q.clone(), i32([1, 1, 1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = esb.esb_cache_attention(q2, c, n2, t, rotation=r)
        held2, _ = esb.esb_cache_attention(q2, c, n2, t, window=50)
    n2.copy_(n)                                                    # lengths are read on the device
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want)
    assert torch.equal(held2, esb.esb_cache_attention(q, c, n, t, window=50)[0])
