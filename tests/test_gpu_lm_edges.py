"""The language-model operators where their calls can go wrong at the edge of
a plan, a buffer or a type: against 64-bit results, with the bounds of
test_gpu_lm.py."""
import pytest
import torch

from paper_2109_03513_gb300 import esb
from test_gpu_lm import TYPES, U, built, close, make_w, matvec_bound, rand, values64  # noqa: F401 (built: a fixture)

pytestmark = pytest.mark.gpu


# the widths whose code stages would fill a ring of three, several tiles a block
@pytest.mark.parametrize("M,N,K,group", [(32, 50000, 2048, 128), (21, 40001, 1537, 128), (24, 39999, 1700, 64), (24, 40000, 4608, 128),
                                         (40, 30001, 4097, 32), (33, 20000, 4500, 64)])
@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16, "codes"])
def test_matvec_many_columns_short_rings(M, N, K, group, x):
    w = make_w(N, K, group, (M + N) % 4)
    rows = rand((M, K), 2)
    if x == "codes":
        rows = esb.esb_project_groups(rows, esb.Fmt(8, 6), 0)[0]
        x64 = values64(rows)
    else:
        rows = rows.to(x)
        x64 = rows.double()
    y = esb.esb_matvec_groups(rows, w, y_dtype=torch.float32)
    w64 = values64(w)
    close(y, x64 @ w64.t(), matvec_bound(x64, w64, K), torch.float32)
    for _ in range(20):
        assert torch.equal(y, esb.esb_matvec_groups(rows, w, y_dtype=torch.float32))
    assert esb.esb_get_status() == 0


# (small, wide; by both kernels) the last row ends its storage, so nothing behind it may be read
@pytest.mark.parametrize("M,N,K,group", [(1, 40, 64, 32), (3, 33, 333, 64), (2, 50, 1000, 0), (4, 200, 4100, 128), (5, 19457, 577, 96),
                                         (40, 16000, 1030, 128)])
def test_matvec_matrix_cut_out_of_a_wider_one(M, N, K, group):
    w = make_w(N, K, group, 2)
    words = -(-K // 32) * 4
    ld = words + 124
    store = torch.randint(-2 ** 31, 2 ** 31 - 1, ((N - 1) * ld + words,), dtype=torch.int32, device="cuda")
    codes = torch.as_strided(store, (N, words), (ld, 1))
    codes.copy_(w.codes[:, :words])
    x = rand((M, K), 3, torch.bfloat16)
    assert torch.equal(esb.esb_matvec_groups(x, esb.Coded(codes, w.scales, w.fmt, K, group)), esb.esb_matvec_groups(x, w))
    assert esb.esb_get_status() == 0


# ------------------------------------------------------------- log probabilities

@pytest.mark.parametrize("rows,cols", [(1, 30000), (2, 200001), (700, 40000), (5, 3000)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [0, 3])
def test_logprobs_nan_stays_whatever_follows(rows, cols, dtype, top):
    # what a thread has met is rescaled by a factor of 0 when a much larger logit follows: a NaN is not lost by it
    part = cols // 2
    good = rand((1, cols), 1, dtype, 3.0).expand(rows, cols)
    ids = torch.full((rows,), cols - 1, dtype=torch.int64, device="cuda")
    want = esb.esb_logprobs(good.contiguous(), ids, top=top)
    assert torch.isfinite(want.lse).all()
    for case in ("block", "one of the masked", "one of the far below", "infinity"):
        x = good.contiguous().clone()
        r = rows // 2
        if case == "block":
            x[r, :part] = float("nan")
        elif case == "one of the masked":
            x[r, :part] = -float("inf")
            x[r, part // 3] = float("nan")
        elif case == "one of the far below":
            x[r, :part] = 0.0
            x[r, part // 3] = float("nan")
            x[r, part:] = 120.0
        else:
            x[r, :part] = -float("inf")
            x[r, part // 3] = float("inf")
        out = esb.esb_logprobs(x, ids, top=top)
        assert torch.isnan(out.lse[r]) and torch.isnan(out.logp[r]) and torch.isnan(out.entropy[r]), case
        others = torch.arange(rows, device="cuda") != r
        assert torch.equal(out.lse[others], want.lse[others]) and torch.equal(out.entropy[others], want.entropy[others])
        if top:
            v = torch.where(torch.isnan(x[r]), torch.full_like(x[r], -float("inf")), x[r]).float()
            assert torch.equal(out.top_ids[r], torch.sort(v, descending=True, stable=True).indices[:top])
        g = torch.ones(rows, device="cuda")
        dx = esb.esb_logprobs_backward(x, ids, out.lse, out.entropy, g, g)
        assert torch.isnan(dx[r]).all() and torch.isfinite(dx[others]).all(), case


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 5000, 40000])
def test_logprobs_from_the_type_s_lowest_to_its_largest(dtype, cols):
    # a difference of two finite logits may be past fp32's range: its probability is 0 and it adds nothing to the entropy
    big = torch.finfo(dtype).max
    x = rand((4, cols), 1, dtype)
    x[0, ::3], x[0, 7] = -big, big
    x[1] = -big
    x[1, cols - 1] = big
    x[2, :] = big
    x[2, 1::2] = -big
    x[3, 5] = big
    ids = torch.tensor([7, cols - 1, 0, 5], device="cuda")
    out = esb.esb_logprobs(x, ids, top=2)
    n = (cols + 1) // 2
    want = torch.tensor([0.0, 0.0, n, 0.0], dtype=torch.float64, device="cuda").clamp_min(1).log()
    # a logarithm and a sum of ones: a few units
    assert ((out.entropy.double() - want).abs() <= 8 * U * (1 + want)).all()
    assert ((out.logp.double() + want).abs() <= 8 * U * (1 + want)).all()
    assert torch.equal(out.top_ids[[0, 1, 3], 0], ids[[0, 1, 3]]) and (out.lse.double() - big).abs().max() <= 2 * U * big + 16
    dx = esb.esb_logprobs_backward(x, ids, out.lse, out.entropy, torch.ones(4, device="cuda"), torch.ones(4, device="cuda"))
    assert torch.isfinite(dx).all()


# ------------------------------------------------------------- other streams

DELAY = 100_000_000                     # clocks that a stream is kept busy, some 50 ms: longer than the host takes for a few calls


def test_backward_workspace_belongs_to_the_call_s_stream():
    # what the current stream allocates after the call is not the workspace that the call's stream has yet to write
    rows, cols = 4096, 1024
    h, dy, w = rand((rows, cols), 1), rand((rows, cols), 2), rand((cols,), 3)
    rstd = esb.esb_rmsnorm(h, None, want_rstd=True).rstd
    dx, dw = torch.empty_like(h), torch.empty(cols, device="cuda")
    want, want_w = esb.esb_rmsnorm_backward(dy, h, w, rstd)
    nb = esb.lib().esb_rmsnorm_backward_workspace_bytes(rows, cols)
    torch.full((1,), 7, dtype=torch.uint8, device="cuda")      # loads what fills below: a load may wait for the device
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(DELAY)
    esb.esb_rmsnorm_backward(dy, h, w, rstd, dx=dx, dweight=dw, stream=st)
    others = [torch.full((nb,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert torch.equal(dx, want) and torch.equal(dw, want_w)
    assert all((t == 7).all() for t in others)


def lm_calls():
    """Each call with the outputs that it makes itself, as a function of the stream."""
    x, r, w, dy = rand((64, 512), 1), rand((64, 512), 2), rand((512,), 3), rand((64, 512), 4)
    m = make_w(128, 512, 64, 2)
    rstd = esb.esb_rmsnorm(x, None, want_rstd=True).rstd
    ids = torch.arange(64, device="cuda")
    lp = esb.esb_logprobs(x, ids)
    return {
        "project": lambda st: [*esb.esb_project_groups(x, esb.Fmt(4, 2), 64, want_xq=True, stream=st)[0][:2],
                               esb.esb_project_groups(x, esb.Fmt(4, 2), 64, want_xq=True, stream=st)[1]],
        "matvec": lambda st: [esb.esb_matvec_groups(x, m, stream=st)],
        "norm": lambda st: (lambda o: [o.h, o.y, o.rstd, *o.coded[:2]])(esb.esb_rmsnorm(x, w, residual=r, want_y=True, want_rstd=True,
                                                                                       fmt=esb.Fmt(8, 6), stream=st)),
        "norm backward": lambda st: list(esb.esb_rmsnorm_backward(dy, x, w, rstd, stream=st)),
        "logprobs": lambda st: list(esb.esb_logprobs(x, ids, top=4, stream=st)),
        "logprobs backward": lambda st: [esb.esb_logprobs_backward(x, ids, lp.lse, None, lp.logp, stream=st)],
    }


@pytest.mark.parametrize("name", ["project", "matvec", "norm", "norm backward", "logprobs", "logprobs backward"])
def test_outputs_belong_to_the_call_s_stream(name):
    # memory that the current stream has yet to write, freed on the host, is not where another stream's outputs go
    call = lm_calls()[name]
    want = [t.clone() for t in call(None)]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(DELAY)
    for t in want:                      # blocks of each output's size, with work waiting on them
        for _ in range(4):
            torch.empty_like(t).fill_(3)
    got = call(st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
