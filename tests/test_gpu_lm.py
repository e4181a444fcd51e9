"""The language-model operators against plain 64-bit implementations: group
projection, matrix-vector products with group scales, RMS norm with its
gradient, log probabilities with theirs.  Codes are compared bit for bit with
the oracle's projection; the tolerances of the rest follow from the number of
fp32 roundings on the way (u = 2^-24 each) and the output type's own."""
import math

import numpy as np
import pytest
import torch

import oracle as o
from paper_2109_03513_gb300 import esb

pytestmark = pytest.mark.gpu

F64 = torch.float64
U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# the rounding of each type: half a unit in the last of its 24, 11 and 8 significant bits, and of its subnormals
HALF = {torch.float32: (U, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(shape, seed, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def close(got, want, abs_err, dtype):
    """|got - want| <= abs_err (a tensor of the fp32 computation's bound) + the output type's rounding."""
    rel, sub = HALF[dtype]
    tol = abs_err + rel * (want.abs() + abs_err) + sub
    d = (got.to(F64) - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), (int(bad.sum()), float((d / tol)[bad].max()))


def unpack(codes, cols, b):
    return o.unpack(codes.cpu().numpy().view(np.uint32), cols, b)


def set_values(b, k):
    return np.array([o.decode(c, b, k) for c in range(1 << b)])


def values64(c: esb.Coded):
    q = set_values(c.fmt.b, c.fmt.k)[unpack(c.codes, c.cols, c.fmt.b)]
    g = c.group if 0 < c.group < c.cols else c.cols
    s = c.scales.double().repeat_interleave(g, 1)[:, :c.cols]
    return torch.as_tensor(q, device="cuda") * s


# ------------------------------------------------------------- projection

def check_projected(coded, xq, x, rounding, scales=None):
    """Every code is the oracle's for the kernel's own scale; every word past the columns holds the zero code."""
    f, (rows, cols) = coded.fmt, x.shape
    g = coded.group if 0 < coded.group < cols else cols
    got = unpack(coded.codes, cols, f.b)
    xn, sn = x.float().cpu().numpy(), coded.scales.cpu().numpy()
    for r in range(rows):
        for j in range(sn.shape[1]):
            part = slice(j * g, min(cols, (j + 1) * g))
            if not np.isfinite(sn[r, j]) or sn[r, j] == 0.0:
                want = np.full(part.stop - part.start, o.zero_code(f.b, f.k))
            else:
                want = o.project_codes(xn[r, part], float(sn[r, j]), f.b, f.k, f.signed, rounding)
            assert np.array_equal(got[r, part], want), (r, j)
    whole = unpack(coded.codes, coded.codes.shape[1] * (32 // f.b), f.b)
    assert (whole[:, cols:] == o.zero_code(f.b, f.k)).all()
    if xq is not None:
        q = torch.as_tensor(set_values(f.b, f.k)[got], dtype=torch.float32, device="cuda")
        want = (coded.scales.repeat_interleave(g, 1)[:, :cols] * q).to(xq.dtype)
        assert torch.equal(torch.nan_to_num(xq, nan=7.0), torch.nan_to_num(want, nan=7.0))


@pytest.mark.parametrize("b,k,signed", [(4, 0, True), (4, 1, True), (4, 2, True), (4, 3, True), (4, 2, False), (8, 6, True),
                                        (8, 3, True), (8, 7, True), (8, 0, True), (8, 2, False)])
@pytest.mark.parametrize("rounding", [0, 1])
def test_project_groups_codes(b, k, signed, rounding):
    for i, (rows, cols, group) in enumerate([(3, 200, 32), (2, 513, 128), (5, 64, 0), (2, 300, 96), (1, 1, 32), (4, 7, 64)]):
        x = rand((rows, cols), 10 * i + k, TYPES[i % 3], std=0.3)
        coded, xq = esb.esb_project_groups(x, esb.Fmt(b, k, signed), group, rounding=rounding, want_xq=True)
        check_projected(coded, xq, x, rounding)
        g = group if 0 < group < cols else cols
        m = x.float().abs() if signed else x.float().clamp_min(0)
        n = -(-cols // g)
        amax = torch.nn.functional.pad(m, (0, n * g - cols)).reshape(rows, n, g).amax(-1).cpu().numpy()
        assert np.array_equal(coded.scales.cpu().numpy(), amax / np.float32(o.C_of(b, k)))


@pytest.mark.parametrize("group", [32, 64, 128, 160, 256, 0])
@pytest.mark.parametrize("b,k", [(4, 2), (8, 6)])
def test_project_groups_ties_and_edges(group, b, k):
    # midpoints of the set with a scale that is a power of two, and their neighbours
    q = np.array(sorted(set_values(b, k)))
    mids = ((q[1:] + q[:-1]) / 2).astype(np.float32)
    row = np.concatenate([mids, np.nextafter(mids, np.float32(9)), np.nextafter(mids, np.float32(-9)), q.astype(np.float32)])
    n = 1024
    x = np.resize(row, n).reshape(1, n).repeat(2, 0) * np.float32(2.0 ** -9)
    x[:, ::32] = np.float32(o.C_of(b, k) * 2.0 ** -9)          # every group reaches the end of the set
    x[1] = -x[1]
    for rounding in (0, 1):
        xd = torch.as_tensor(x, device="cuda")
        coded, xq = esb.esb_project_groups(xd, esb.Fmt(b, k), group, rounding=rounding, want_xq=True)
        assert (coded.scales == 2.0 ** -9).all()
        check_projected(coded, xq, xd, rounding)


@pytest.mark.parametrize("rule", [esb.ESB_SCALE_ABSMAX, esb.ESB_SCALE_DDA])
def test_project_groups_special_values(rule):
    x = rand((10, 256), 3)
    x[0] = 0.0
    x[1, 5] = float("nan")
    x[2, 200] = float("inf")
    x[3, 7] = -float("inf")
    x[4] *= 1e-42                                                # subnormal scale
    x[5] *= 3e37
    x[6, 64:128] = 0.0
    x[7] = 1e-45
    x[8] = -0.0
    for f in (esb.Fmt(4, 2), esb.Fmt(8, 6)):
        coded, xq = esb.esb_project_groups(x, f, 64, rule=rule, want_xq=True)
        check_projected(coded, xq, x, 0)
        s = coded.scales
        if rule == esb.ESB_SCALE_ABSMAX:
            assert (s[0] == 0).all() and s[6, 1] == 0 and (s[8] == 0).all() and torch.isinf(s[2, 3]) and torch.isinf(s[3, 0])
        assert torch.isnan(s[1, 0]) and torch.isfinite(s[1, 1:]).all()
        assert torch.isnan(xq[1, :64]).all() and torch.isnan(xq[2, 192:]).all() and torch.isfinite(xq[2, :192]).all()


@pytest.mark.parametrize("b,k,signed", [(4, 2, True), (4, 1, True), (8, 6, False)])
@pytest.mark.parametrize("group,cols", [(32, 128), (128, 1000), (0, 4096), (96, 333)])
def test_project_groups_dda_scale(b, k, signed, group, cols):
    x = rand((6, cols), cols, torch.float32, 0.7) + 0.4
    coded, _ = esb.esb_project_groups(x, esb.Fmt(b, k, signed), group, rule=esb.ESB_SCALE_DDA)
    check_projected(coded, None, x, 0)
    g = group if 0 < group < cols else cols
    a = esb.esb_alpha_star(b, k)[0]
    for j in range(coded.scales.shape[1]):
        p = x[:, j * g:(j + 1) * g].double()
        n = p.shape[1]
        spread = ((p - p.mean(1, keepdim=True)) if signed else p).square().mean(1).sqrt()
        want = a * (spread + 1e-7)
        # sums of n terms in fp32 (each lane's, then a tree), half of the relative error through the root;
        # the mean's error enters squared; alpha* rounded, the root, the sum and the product
        tol = ((n / 256 + 16) / 2 + 6) * U
        assert ((coded.scales[:, j].double() - want).abs() <= tol * want).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_project_groups_strides_and_offsets(dtype):
    # rows of a wider matrix, starting at odd places, into code rows with room to spare
    base = rand((9, 1111), 5, dtype)
    x = base[1:8, 3:3 + 777]
    codes = torch.full((7, 140), -1, dtype=torch.int32, device="cuda")
    wide = torch.zeros((7, 900), dtype=dtype, device="cuda")
    coded, xq = esb.esb_project_groups(x, esb.Fmt(4, 1), 64, codes=codes, xq=wide[:, 5:782])
    check_projected(coded, xq, x, 0)
    ref, _ = esb.esb_project_groups(x.contiguous(), esb.Fmt(4, 1), 64)
    assert torch.equal(ref.codes[:, :98], codes[:, :98]) and torch.equal(ref.scales, coded.scales)
    assert (wide[:, :5] == 0).all() and (wide[:, 782:] == 0).all()


def test_project_groups_random_quotients_are_ieee():
    # the division by a common scale against numpy's, over many scales and magnitudes (codes with the most significant bits)
    g = gen(11)
    x = torch.exp2(torch.rand((4096, 64), generator=g, device="cuda") * 8 - 8) * torch.rand((4096, 1), generator=g, device="cuda").add(0.5)
    coded, _ = esb.esb_project_groups(x, esb.Fmt(8, 7), 32)
    check_projected(coded, None, x, 0)


# ------------------------------------------------------------- matvec

def make_w(n, k, group, fk, seed=1):
    return esb.esb_project_groups(rand((n, k), seed, std=0.1), esb.Fmt(4, fk), group)[0]


def matvec_bound(x64, w64, K):
    """fp32 bound of a sum of K products in any order of the kernel's: at most 32 + K / 128 roundings (twice a unit each
    where a matrix instruction cuts) on every term's way, and an input's bits below 2^-39 of its 128 neighbours' largest."""
    s = x64.abs() @ w64.abs().t()
    tail = K * 2.0 ** -39 * x64.abs().amax(1, keepdim=True) * w64.abs().amax(1)[None]
    return (32 + K / 128) * 2 * U * s + tail


@pytest.mark.parametrize("M,N,K,group", [(1, 1, 1, 0), (1, 17, 32, 32), (1, 300, 576, 64), (2, 64, 1000, 128), (3, 130, 4096, 128),
                                         (5, 33, 777, 32), (8, 100, 513, 96), (16, 48, 2048, 0), (17, 257, 1030, 64),
                                         (33, 70, 384, 160), (64, 129, 2176, 256), (1, 4096, 9216, 128), (7, 40, 20000, 32),
                                         (130, 24, 640, 128)])
@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_matches_fp64(M, N, K, group, dtype):
    w = make_w(N, K, group, (M + N) % 4)
    x = rand((M, K), 2, dtype)
    w64, x64 = values64(w), x.double()
    y = esb.esb_matvec_groups(x, w)
    assert y.dtype == dtype
    close(y, x64 @ w64.t(), matvec_bound(x64, w64, K), dtype)


@pytest.mark.parametrize("M,N,K,group,xgroup", [(1, 40, 96, 32, 0), (4, 64, 9216, 64, 0), (9, 65, 513, 128, 0), (3, 50, 1024, 128, 256),
                                                (2, 31, 1000, 32, 64), (20, 20, 700, 0, 0), (1, 16, 1, 0, 0), (5, 40, 384, 96, 96)])
@pytest.mark.parametrize("xk", [2, 3, 6, 7])
def test_matvec_coded_rows(M, N, K, group, xgroup, xk):
    w = make_w(N, K, group, xk % 4)
    xc = esb.esb_project_groups(rand((M, K), 4), esb.Fmt(8, xk, xk != 3), xgroup)[0]
    w64, x64 = values64(w), values64(xc)
    bias = rand((N,), 8)
    y = esb.esb_matvec_groups(xc, w, bias=bias, y_dtype=torch.float32)
    want = x64 @ w64.t() + bias.double()
    close(y, want, matvec_bound(x64, w64, K) + U * want.abs(), torch.float32)
    assert esb.esb_matvec_groups(xc, w).dtype == torch.bfloat16


# enough matrix rows for every SM to get tiles of 128
@pytest.mark.parametrize("M,N,K,group", [(1, 16384, 512, 128), (1, 15700, 1000, 64), (2, 20001, 64, 32), (5, 19457, 577, 96),
                                         (8, 30000, 33, 0), (16, 15616, 4096, 128), (17, 16000, 2050, 256), (32, 40000, 300, 64),
                                         (40, 15999, 1024, 32), (3, 60000, 130, 128), (24, 16000, 700, 128), (12, 20000, 513, 96),
                                         (33, 15616, 4096, 128)])
@pytest.mark.parametrize("x", [torch.float32, torch.float16, torch.bfloat16, "codes"])
def test_matvec_many_columns(M, N, K, group, x):
    w = make_w(N, K, group, (M + N) % 4)
    rows = rand((M, K), 2)
    if x == "codes":
        rows = esb.esb_project_groups(rows, esb.Fmt(8, 6), 0)[0]
        x64 = values64(rows)
    else:
        rows = rows.to(x)
        x64 = rows.double()
    bias = rand((N,), 3)
    out = torch.full((M, N + 3), 5.0, dtype=torch.float32, device="cuda")
    y = esb.esb_matvec_groups(rows, w, bias=bias, y=out[:, 1:N + 1])
    w64 = values64(w)
    want = x64 @ w64.t() + bias.double()
    close(y, want, matvec_bound(x64, w64, K) + U * want.abs(), torch.float32)
    assert (out[:, 0] == 5).all() and (out[:, N + 1:] == 5).all()
    assert torch.equal(y, esb.esb_matvec_groups(rows, w, bias=bias, y_dtype=torch.float32))
    assert esb.esb_get_status() == 0


# few matrix rows, long ones
@pytest.mark.parametrize("M,N,K,group", [(4, 1, 4096, 128), (4, 4096, 4096, 64), (5, 1000, 4097, 32), (8, 33, 5121, 96), (16, 2000, 9216, 128),
                                         (6, 9700, 9728, 128), (31, 17, 6655, 64), (100, 300, 4608, 0), (3, 500, 14336, 32)])
@pytest.mark.parametrize("x", [torch.float32, torch.float16, torch.bfloat16, "codes"])
def test_matvec_long_rows(M, N, K, group, x):
    w = make_w(N, K, group, (M + N) % 4)
    rows = rand((M, K), 2)
    if x == "codes":
        rows = esb.esb_project_groups(rows, esb.Fmt(8, 5), 2 * group)[0]
        x64 = values64(rows)
    else:
        rows = rows.to(x)
        x64 = rows.double()
    bias = rand((N,), 3)
    y = esb.esb_matvec_groups(rows, w, bias=bias, y_dtype=torch.float32)
    w64 = values64(w)
    want = x64 @ w64.t() + bias.double()
    close(y, want, matvec_bound(x64, w64, K) + U * want.abs(), torch.float32)
    assert torch.equal(y, esb.esb_matvec_groups(rows, w, bias=bias, y_dtype=torch.float32))


def test_matvec_many_columns_special_values_and_padding():
    K, N = 333, 16001
    x = rand((5, K), 9)
    x[0, 3] = float("inf")
    x[1, 200] = float("nan")
    x[3] = 0
    x[4, 100] = -float("inf")
    w = esb.esb_project_groups(rand((N, K), 3).abs() + 0.5, esb.Fmt(4, 2), 64)[0]     # no zero weight
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (N, 48), dtype=torch.int32, device="cuda")
    codes[:, :42] = w.codes[:, :42]
    scales = torch.full((N, 9), float("nan"), device="cuda")
    scales[:, :6] = w.scales
    y = esb.esb_matvec_groups(x, esb.Coded(codes, scales[:, :6], w.fmt, K, 64))
    assert (y[0] == float("inf")).all() and torch.isnan(y[1]).all() and (y[3] == 0).all() and (y[4] == -float("inf")).all()
    close(y[2:3], x[2:3].double() @ values64(w).t(), matvec_bound(x[2:3].double(), values64(w), K), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_wide_range_rows(dtype):
    # values over the whole of the type's range, in blocks of their own size
    K = 1024
    x = rand((4, K), 6)
    top = {torch.float32: 60, torch.bfloat16: 60, torch.float16: 6}[dtype]
    e = torch.randint(-top, top, (4, K // 128), generator=gen(7), device="cuda").float().repeat_interleave(128, 1)
    x = (x * torch.exp2(e)).to(dtype)
    w = make_w(96, K, 128, 1)
    w64, x64 = values64(w), x.double()
    y = esb.esb_matvec_groups(x, w, y_dtype=torch.float32)
    close(y, x64 @ w64.t(), matvec_bound(x64, w64, K), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_special_values(dtype):
    K = 256
    x = rand((5, K), 9, dtype)
    big = torch.finfo(dtype).max
    x[0, 3] = float("inf")
    x[1, 200] = float("nan")
    x[2, 7] = big
    x[3] = 0
    x[4, 100] = -float("inf")
    # no zero weight, and sums of the type's largest value that fp32 still holds
    w = esb.esb_project_groups((rand((40, K), 3).abs() + 0.5) / 16, esb.Fmt(4, 2), 64)[0]
    y = esb.esb_matvec_groups(x, w, y_dtype=torch.float32).double()
    assert (y[0] == float("inf")).all() and torch.isnan(y[1]).all() and (y[3] == 0).all() and (y[4] == -float("inf")).all()
    want = x[2:3].double() @ values64(w).t()
    close(y[2:3].float(), want, matvec_bound(x[2:3].double(), values64(w), K), torch.float32)
    # a group that holds a NaN weight gives NaN
    wr = rand((40, K), 3)
    wr[7, 70] = float("nan")
    w = esb.esb_project_groups(wr, esb.Fmt(4, 2), 64)[0]
    y = esb.esb_matvec_groups(rand((2, K), 1, dtype), w)
    assert torch.isnan(y[:, 7]).all() and torch.isfinite(y[:, :7]).all() and torch.isfinite(y[:, 8:]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_strides_and_padding(dtype):
    # rows of a wider matrix at odd offsets; code rows longer than the columns, garbage (and NaN scales) behind them
    K, N, M = 333, 50, 6
    w = make_w(N, K, 64, 2)
    codes = torch.randint(-2 ** 31, 2 ** 31 - 1, (N, 64), dtype=torch.int32, device="cuda")
    codes[:, :42] = w.codes[:, :42]
    scales = torch.full((N, 11), float("nan"), device="cuda")
    scales[:, :6] = w.scales
    wide = rand((M + 1, 700), 5, dtype)
    x = wide[1:, 7:7 + K]
    out = torch.full((M, 99), 5.0, dtype=dtype, device="cuda")
    y = esb.esb_matvec_groups(x, esb.Coded(codes, scales[:, :6], w.fmt, K, 64), y=out[:, 3:53])
    assert torch.equal(y, esb.esb_matvec_groups(x.contiguous(), w))
    assert (out[:, :3] == 5).all() and (out[:, 53:] == 5).all()


def test_matvec_offsets_past_32_bits():
    # a matrix whose last rows lie past 2^32 words
    K, N = 64, 3
    ld = (1 << 31) + 4
    w = make_w(N, K, 32, 2)
    store = torch.empty((N - 1) * ld + 8, dtype=torch.int32, device="cuda")
    codes = torch.as_strided(store, (N, 8), (ld, 1))
    codes.copy_(w.codes)
    x = rand((2, K), 3)
    assert torch.equal(esb.esb_matvec_groups(x, esb.Coded(codes, w.scales, w.fmt, K, 32)), esb.esb_matvec_groups(x, w))


def test_matvec_repeats_bit_for_bit_and_on_another_stream():
    w = make_w(513, 2050, 128, 2)
    x = rand((3, 2050), 1, torch.bfloat16)
    want = esb.esb_matvec_groups(x, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        y = torch.empty_like(want)
        esb.esb_matvec_groups(x, w, y=y, stream=st)
        st.synchronize()
        assert torch.equal(y, want)


# ------------------------------------------------------------- norm

def norm64(x, r, w, eps):
    z = x.double() + (r.double() if r is not None else 0.0)
    rstd = 1.0 / (z.square().mean(1, keepdim=True) + eps).sqrt()
    return z, rstd, z * rstd * (w.double() if w is not None else 1.0)


def norm_bound(y, cols):
    """Roundings of y: the sum and the products, and rstd's (its mean of squares counts half: a thread's part of the
    row in turn, then trees of partial sums)."""
    return (8 + (cols / 256 + 24) / 2) * U * y.abs()


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 128), (2, 1000), (4, 1025), (2, 8192), (3, 16384), (1, 40000), (300, 64), (37, 2050)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_rmsnorm_matches_fp64(rows, cols, dtype):
    for i, (res, wt) in enumerate([(True, dtype), (False, torch.float32), (True, None)]):
        x, r = rand((rows, cols), 1 + i, dtype), rand((rows, cols), 2 + i, dtype, 3.0) if res else None
        w = rand((cols,), 3, wt) if wt else None
        out = esb.esb_rmsnorm(x, w, 1e-5, residual=r, want_rstd=True)
        z, rstd, y = norm64(x, r, w, 1e-5)
        close(out.y, y, norm_bound(y, cols), dtype)
        close(out.rstd, rstd[:, 0], norm_bound(rstd[:, 0], cols), torch.float32)
        if res:
            assert torch.equal(out.h, (x.float() + r.float()).to(dtype))
        assert out.coded is None and out.yq is None


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("group", [0, 32, 64, 96, 128, 512])
def test_rmsnorm_codes(rows, cols, group):
    if rows * -(-cols // (group or cols)) > 1500:
        rows = 3
    for i, (b, k, signed, rounding) in enumerate([(8, 6, True, 0), (8, 3, True, 1), (8, 6, False, 0), (8, 0, True, 0)]):
        dtype = TYPES[(i + cols) % 3]
        x, r, w = rand((rows, cols), 4, dtype), rand((rows, cols), 5, dtype), rand((cols,), 6, dtype)
        yq = torch.empty((rows, cols), dtype=torch.float32, device="cuda")
        out = esb.esb_rmsnorm(x, w, 1e-6, residual=r, fmt=esb.Fmt(b, k, signed), group=group, rounding=rounding, yq=yq,
                              want_y=True, y_dtype=torch.float32)
        _, _, y = norm64(x, r, w, 1e-6)
        close(out.y, y, norm_bound(y, cols), torch.float32)
        assert torch.equal(out.h, (x.float() + r.float()).to(dtype))
        # the codes are those of the fp32 norm, with scales that it fixes
        check_projected(out.coded, out.yq, out.y, rounding)
        g = group if 0 < group < cols else cols
        n = -(-cols // g)
        m = out.y.abs() if signed else out.y.clamp_min(0)
        amax = torch.nn.functional.pad(m, (0, n * g - cols)).reshape(rows, n, g).amax(-1).cpu().numpy()
        assert np.array_equal(out.coded.scales.cpu().numpy(), amax / np.float32(o.C_of(b, k)))
        # without the other outputs the same codes
        only = esb.esb_rmsnorm(x, w, 1e-6, residual=r, fmt=esb.Fmt(b, k, signed), group=group, rounding=rounding)
        assert only.y is None and torch.equal(only.coded.codes, out.coded.codes) and torch.equal(only.coded.scales, out.coded.scales)


def test_rmsnorm_special_values():
    x = rand((5, 512), 1)
    x[0] = 0.0
    x[1, 3] = float("nan")
    x[2, 9] = float("inf")
    x[3] *= 1e-22
    out = esb.esb_rmsnorm(x, None, 0.0, fmt=esb.Fmt(8, 6), group=128, want_y=True)
    assert torch.isnan(out.y[0]).all() and torch.isnan(out.y[1]).all()
    assert torch.isnan(out.y[2, 9]) and (out.y[2, :9] == 0).all()
    out = esb.esb_rmsnorm(x, None, 1e-6, fmt=esb.Fmt(8, 6), group=128, want_y=True)
    assert (out.y[0] == 0).all() and (out.coded.scales[0] == 0).all()
    check_projected(out.coded, None, out.y, 0)
    _, _, y = norm64(x[3:], None, None, 1e-6)
    close(out.y[3:], y, norm_bound(y, 512), torch.float32)


@pytest.mark.parametrize("cols", [512, 515, 33000])
@pytest.mark.parametrize("group", [None, 0, 64])
def test_rmsnorm_in_place_and_strided(cols, group):
    fmt = None if group is None else esb.Fmt(8, 6)
    x, r, w = rand((9, cols), 1, torch.bfloat16), rand((9, cols + 3), 2, torch.bfloat16)[:, 1:cols + 1], rand((cols,), 3)
    kw = dict(fmt=fmt, group=group or 0, want_y=True)
    want = esb.esb_rmsnorm(x, w, residual=r.contiguous(), **kw)
    r2 = r.clone(memory_format=torch.preserve_format)
    x2 = x.clone()
    got = esb.esb_rmsnorm(x2, w, residual=r2, h=r2, y=x2, **kw)
    assert torch.equal(got.h, want.h) and torch.equal(got.y, want.y) and got.y.data_ptr() == x2.data_ptr()
    if fmt:
        assert torch.equal(got.coded.codes, want.coded.codes)
    wide = torch.full((9, cols + 20), 3.0, dtype=torch.bfloat16, device="cuda")
    esb.esb_rmsnorm(x, w, residual=r, y=wide[:, 9:9 + cols], **kw)
    assert torch.equal(wide[:, 9:9 + cols], want.y) and (wide[:, :9] == 3).all() and (wide[:, 9 + cols:] == 3).all()


def grad64(dy, h, w, rstd, dh):
    n, d = h.double() * rstd.double()[:, None], dy.double() * (w.double() if w is not None else 1.0)
    m = (d * n).mean(1, keepdim=True)
    dx = rstd.double()[:, None] * (d - n * m) + (dh.double() if dh is not None else 0.0)
    return dx, (dy.double() * n).sum(0), n, d, m


@pytest.mark.parametrize("rows,cols", SHAPES + [(1000, 520), (4099, 96)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rmsnorm_backward_matches_fp64(rows, cols, dtype):
    for i, (wt, dh, gt) in enumerate([(dtype, True, dtype), (torch.float32, False, torch.float32), (None, True, dtype)]):
        h, dy = rand((rows, cols), 1, dtype), rand((rows, cols), 2, gt, 0.01)
        w, dhv = rand((cols,), 3, wt) if wt else None, rand((rows, cols), 4, dtype, 0.01) if dh else None
        rstd = esb.esb_rmsnorm(h, None, 1e-6, want_rstd=True).rstd
        dx, dw = esb.esb_rmsnorm_backward(dy, h, w, rstd, dh=dhv, want_dweight=True)
        want, want_dw, n, d, m = grad64(dy, h, w, rstd, dhv)
        # the row's mean: its terms' sum (a thread's part in turn, then trees); then a few roundings of each term
        em = (cols / 256 + 32) * U * (d * n).abs().mean(1, keepdim=True)
        rs = rstd.double()[:, None]
        err = rs * (6 * U * (d.abs() + (n * m).abs()) + n.abs() * em) + 2 * U * want.abs()
        close(dx, want, err, dtype)
        # dweight: sums over the rows in chains, then over the parts
        err = (rows + 8) * U * (dy.double() * n).abs().sum(0)
        close(dw, want_dw, err, torch.float32)
        only, none = esb.esb_rmsnorm_backward(dy, h, w, rstd, dh=dhv, want_dweight=False)
        assert none is None and torch.equal(only, dx)


def test_rmsnorm_backward_against_differences():
    # central differences of sum(g * y(x)) in 64 bits at h = 1e-5: truncation h^2, roundings 1e-16 / h
    rows, cols, eps = 3, 40, 1e-3
    x, w, g = rand((rows, cols), 1), rand((cols,), 2), rand((rows, cols), 3)
    out = esb.esb_rmsnorm(x, w, eps, want_rstd=True)
    dx, dw = esb.esb_rmsnorm_backward(g, x, w, out.rstd)
    f = lambda x, w: (g.double() * norm64(x, None, w, eps)[2]).sum()
    for idx in [(0, 0), (1, 17), (2, 39)]:
        e = torch.zeros((rows, cols), dtype=F64, device="cuda")
        e[idx] = 1e-5
        d = (f(x.double() + e, w) - f(x.double() - e, w)) / 2e-5
        assert abs(float(d) - float(dx[idx])) <= 1e-5 * (1 + abs(float(d)))
    for j in (0, 21):
        e = torch.zeros(cols, dtype=F64, device="cuda")
        e[j] = 1e-5
        d = (f(x, w.double() + e) - f(x, w.double() - e)) / 2e-5
        assert abs(float(d) - float(dw[j])) <= 1e-5 * (1 + abs(float(d)))


def test_rmsnorm_backward_in_place_and_strided():
    h, dy, dh, w = (rand(s, i, torch.bfloat16) for i, s in enumerate([(20, 515), (20, 515), (20, 515), (515,)]))
    rstd = esb.esb_rmsnorm(h, None, want_rstd=True).rstd
    dx, dw = esb.esb_rmsnorm_backward(dy, h, w, rstd, dh=dh)
    for other in (dy, h, dh):
        args = [t.clone() if t is other else t for t in (dy, h, dh)]
        into = args[[dy is other, h is other, dh is other].index(True)]
        got, gw = esb.esb_rmsnorm_backward(args[0], args[1], w, rstd, dh=args[2], dx=into)
        assert torch.equal(got, dx) and torch.equal(gw, dw)
    wide = [torch.zeros((20, 600), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    for t, v in zip(wide, (dy, h, dh)):
        t[:, 3:518] = v
    got, gw = esb.esb_rmsnorm_backward(*(t[:, 3:518] for t in wide[:2]), w, rstd, dh=wide[2][:, 3:518], dx=wide[3][:, 3:518])
    assert torch.equal(got, dx) and torch.equal(gw, dw) and (wide[3][:, :3] == 0).all() and (wide[3][:, 518:] == 0).all()


# ------------------------------------------------------------- log probabilities

def lp64(x, ids):
    x = x.double()
    lse = torch.logsumexp(x, 1)
    logp = x - lse[:, None]
    p = logp.exp()
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    ok = (ids >= 0) & (ids < x.shape[1])
    lp = torch.where(ok, logp.gather(1, torch.where(ok, ids, 0)[:, None])[:, 0], torch.zeros_like(lse))
    return lse, lp, ent, p, logp


# exp of a difference d carries about 2 + 1.16 |d| units (2^-23) on a term e^d, so the sum's relative error stays
# under the weighted mean of those, (2 + 1.16 (H + 1)) 2^-23 with d's mean below the entropy H <= 12 + 1; the trees of
# partial sums add a few dozen roundings at most
LSE_ERR = (2 + 1.16 * 14 + 40) * 2.0 ** -23


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (2, 33), (7, 1000), (2, 4097), (3, 32768), (1, 131072), (2, 200001), (1, 400000),
                                       (200, 129), (50, 5000)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [0, 1, 8, 32])
def test_logprobs_matches_fp64(rows, cols, dtype, top):
    x = rand((rows, cols), cols % 97, dtype, 3.0)
    if cols > 8:
        x[:, cols // 2: cols // 2 + cols // 8] = -float("inf")
    ids = torch.randint(0, cols, (rows,), generator=gen(2), device="cuda")
    if rows > 2:
        ids[1], ids[2] = -100, cols
    out = esb.esb_logprobs(x, ids, top=top)
    lse, lp, ent, _, _ = lp64(x, ids)
    fin = torch.isfinite(lp)
    assert torch.equal(torch.isfinite(out.logp), fin)
    close(out.lse, lse, LSE_ERR + 2 * U * lse.abs(), torch.float32)
    close(out.logp[fin], lp[fin], LSE_ERR + 4 * U * (lp[fin].abs() + 30), torch.float32)
    close(out.entropy, ent, LSE_ERR * (2 + ent.abs()) * 2, torch.float32)
    if top:
        n = min(top, cols)
        want = torch.sort(x.float(), dim=1, descending=True, stable=True)
        v, i = want.values[:, :n], want.indices[:, :n]
        real = v > -float("inf")
        assert torch.equal(out.top_ids[:, :n], torch.where(real, i, -1))
        assert (out.top_ids[:, n:] == -1).all() and (out.top_logp[:, n:] == -float("inf")).all()
        assert (out.top_logp[:, :n][~real] == -float("inf")).all()
        t = (v.double() - lse[:, None])[real]
        close(out.top_logp[:, :n][real], t, LSE_ERR + 4 * U * (t.abs() + 30), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [5, 1000, 40000, 131072])
def test_logprobs_ties_and_few_values(dtype, cols):
    # all equal; two values only; ascending; a few unmasked; the largest at the very end
    x = torch.zeros((6, cols), dtype=dtype, device="cuda")
    x[1, ::3] = 1.0
    x[2] = (torch.arange(cols, device="cuda") * (60.0 / cols)).to(dtype)
    x[3] = -float("inf")
    x[3, cols // 2], x[3, cols - 1], x[3, 0] = 2.0, 2.0, -1.0
    x[4, -1] = 9.0
    x[5, : cols // 2] = -0.0
    out = esb.esb_logprobs(x, None, top=20)
    n = min(20, cols)
    v, i = torch.sort(x.float(), dim=1, descending=True, stable=True)
    want = torch.where(v > -float("inf"), i, -1)[:, :n]
    assert torch.equal(out.top_ids[:, :n], want)
    assert out.logp is None
    lse, _, ent, _, _ = lp64(x, torch.zeros(6, dtype=torch.int64, device="cuda"))
    close(out.lse, lse, LSE_ERR + 2 * U * lse.abs(), torch.float32)
    close(out.entropy, ent, LSE_ERR * (2 + ent.abs()) * 2, torch.float32)


@pytest.mark.parametrize("rows,cols", [(1, 150001), (2, 60000), (700, 20000)])
@pytest.mark.parametrize("top", [1, 13, 32])
def test_logprobs_alternatives_of_ascending_rows(rows, cols, top):
    # every logit is an alternative when it is met: more candidates than a list of them holds
    x = (torch.arange(cols, device="cuda") * 2.0 ** -16).repeat(rows, 1)
    x[:, cols // 3: cols // 3 + 50] = float("nan") if rows == 2 else -float("inf")
    x[rows // 2, 5] = 7.0
    out = esb.esb_logprobs(x, None, top=top)
    v = torch.where(torch.isnan(x), torch.full_like(x, -float("inf")), x)
    assert torch.equal(out.top_ids, torch.sort(v, dim=1, descending=True, stable=True).indices[:, :top])


@pytest.mark.parametrize("cols", [3, 700, 70000])
def test_logprobs_empty_and_special_rows(cols):
    x = rand((6, cols), 1)
    x[0] = -float("inf")
    x[1, cols // 2] = float("nan")
    x[2, cols - 1] = float("inf")
    x[3] = torch.finfo(torch.float32).min                        # masks of the type's lowest value
    x[3, 1] = 0.25
    x[4] = float("nan")
    ids = torch.ones(6, dtype=torch.int64, device="cuda")
    out = esb.esb_logprobs(x, ids, top=2)
    assert out.lse[0] == -float("inf") and out.logp[0] == -float("inf") and out.entropy[0] == 0
    assert (out.top_ids[0] == -1).all() and (out.top_logp[0] == -float("inf")).all()
    for r in (1, 2, 4):
        assert torch.isnan(out.lse[r]) and torch.isnan(out.logp[r]) and torch.isnan(out.entropy[r])
    assert (out.top_ids[4] == -1).all()
    best = torch.where(torch.isnan(x[1]), torch.full_like(x[1], -float("inf")), x[1]).argmax()
    assert out.top_ids[1, 0] == best and out.top_ids[2, 0] == cols - 1
    assert out.lse[3] == 0.25 and out.logp[3] == 0 and out.entropy[3] == 0 and out.top_ids[3, 0] == 1 and out.top_ids[3, 1] == 0
    gl, gh = torch.ones(6, device="cuda"), torch.ones(6, device="cuda")
    dx = esb.esb_logprobs_backward(x, ids, out.lse, out.entropy, gl, gh)
    assert (dx[0, :1] == 0).all() and (dx[0, 2:] == 0).all()
    assert (dx[3] == 0).all()                                    # p = 1 at the id: its own gradient is 1 - p = 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 3), (3, 129), (40, 4097), (2, 131072), (7, 50001)])
def test_logprobs_backward_matches_fp64(rows, cols, dtype):
    x = rand((rows, cols), 7, dtype, 3.0)
    if cols > 8:
        x[:, ::7] = -float("inf")
    ids = torch.randint(0, cols, (rows,), generator=gen(2), device="cuda")
    if rows > 2:
        ids[1] = -1
    gl, gh = rand((rows,), 1), rand((rows,), 2)
    out = esb.esb_logprobs(x, ids)
    _, _, _, p, _ = lp64(x, ids)
    lse, ent = out.lse.double()[:, None], out.entropy.double()[:, None]
    lp = x.double() - lse
    pk = lp.exp()
    ok = ((ids >= 0) & (ids < cols)).double()[:, None]
    one = torch.zeros_like(pk).scatter_(1, ids.clamp(0, cols - 1)[:, None], 1.0) * ok
    for a, b in ((gl, gh), (gl, None), (None, gh)):
        got = esb.esb_logprobs_backward(x, ids, out.lse, out.entropy, a, b)
        g1 = a.double()[:, None] * ok if a is not None else torch.zeros_like(lse)
        g2 = b.double()[:, None] if b is not None else torch.zeros_like(lse)
        in_h = torch.where(pk > 0, pk * (lp + ent), torch.zeros_like(pk))
        want = g1 * (one - pk) - g2 * in_h
        # x - lse rounded (its error moves p by that much), exp's own units, and the products
        ep = pk * ((lp.nan_to_num(neginf=0.0).abs() * (1.16 * 2 + 1) + 8) * 2 * U)
        err = (g1.abs() + g2.abs() * (lp.nan_to_num(neginf=0.0).abs() + ent + 1)) * ep + 4 * U * (want.abs() + g1.abs() * one) + 2.0 ** -126
        close(got, want, err, dtype)
        assert (got[torch.isinf(x) & (one == 0)] == 0).all()


def test_logprobs_backward_against_differences():
    # central differences of sum(gl logp + gh H) in 64 bits at 1e-5
    rows, cols = 3, 50
    x, gl, gh = rand((rows, cols), 1, std=2.0), rand((rows,), 2), rand((rows,), 3)
    ids = torch.tensor([4, 49, -100], device="cuda")
    out = esb.esb_logprobs(x, ids)
    dx = esb.esb_logprobs_backward(x, ids, out.lse, out.entropy, gl, gh)

    def f(x):
        _, lp, ent, _, _ = lp64(x, ids)
        return (gl.double() * lp + gh.double() * ent).sum()

    for idx in [(0, 4), (0, 9), (1, 49), (1, 0), (2, 7)]:
        e = torch.zeros((rows, cols), dtype=F64, device="cuda")
        e[idx] = 1e-5
        d = (f(x.double() + e) - f(x.double() - e)) / 2e-5
        assert abs(float(d) - float(dx[idx])) <= 1e-5 * (1 + abs(float(d)))


@pytest.mark.parametrize("dtype", TYPES)
def test_logprobs_strides_offsets_in_place(dtype):
    wide = rand((9, 6011), 3, dtype)
    x = wide[2:8, 5:5 + 5001]
    ids = torch.randint(0, 5001, (6,), generator=gen(1), device="cuda")
    a, b = esb.esb_logprobs(x, ids, top=5), esb.esb_logprobs(x.contiguous(), ids, top=5)
    assert torch.equal(a.top_ids, b.top_ids)
    close(a.lse, b.lse.double(), 2 * LSE_ERR + 4 * U * b.lse.abs().double(), torch.float32)
    gl = rand((6,), 1)
    before = wide.clone()
    want = esb.esb_logprobs_backward(x, ids, a.lse, None, gl)
    got = esb.esb_logprobs_backward(x, ids, a.lse, None, gl, dlogits=x)
    assert torch.equal(got, want)
    assert torch.equal(wide[:2], before[:2]) and torch.equal(wide[:, :5], before[:, :5]) and torch.equal(wide[:, 5006:], before[:, 5006:])


def test_logprobs_offsets_past_32_bits():
    ld, cols = (1 << 31) + 1, 1000
    store = torch.empty(2 * ld + cols, dtype=torch.float16, device="cuda")
    x = torch.as_strided(store, (3, cols), (ld, 1))
    x.copy_(rand((3, cols), 1, torch.float16))
    ids = torch.tensor([1, 2, 999], device="cuda")
    a, b = esb.esb_logprobs(x, ids, top=3), esb.esb_logprobs(x.contiguous(), ids, top=3)
    assert torch.equal(a.top_ids, b.top_ids)
    close(a.logp, b.logp.double(), 2 * LSE_ERR + 40 * U, torch.float32)


def test_logprobs_repeats_bit_for_bit_and_on_another_stream():
    x = rand((3, 70001), 5, torch.bfloat16, 3.0)
    ids = torch.tensor([5, 6, 7], device="cuda")
    want = esb.esb_logprobs(x, ids, top=10)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        got = esb.esb_logprobs(x, ids, top=10, stream=st)
        st.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------- sizes of nothing

def test_empty_tensors():
    for rows, cols in ((0, 64), (0, 0)):
        x = torch.empty((rows, cols), device="cuda")
        esb.esb_project_groups(x, esb.Fmt(4, 2), 32)
        esb.esb_rmsnorm(x, None, fmt=esb.Fmt(8, 6))
        esb.esb_logprobs(x, None)
    x = torch.empty((0, 64), device="cuda")
    _, dw = esb.esb_rmsnorm_backward(x, x, None, torch.empty(0, device="cuda"), want_dweight=True)
    assert (dw == 0).all()
    w = make_w(10, 64, 32, 2)
    assert esb.esb_matvec_groups(x, w).shape == (0, 10)
    assert esb.esb_get_status() == 0
