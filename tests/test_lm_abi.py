"""Refusals of the language-model operators: host-side validation of the C ABI
and of the binding (no device work; runs without a GPU)."""
import ctypes

import pytest
import torch

from paper_2109_03513_gb300 import esb

P = ctypes.c_void_p(256)            # an aligned address that nothing reads: every call here is refused, or has nothing to do
ODD = ctypes.c_void_p(257)
INV, UNS, RNG, ALN = esb.ESB_ERR_INVALID_ARG, esb.ESB_ERR_UNSUPPORTED, esb.ESB_ERR_RANGE, esb.ESB_ERR_ALIGN


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    return esb.lib()


F4, F8 = esb.Fmt(4, 2).c(), esb.Fmt(8, 6).c()


def project(lib, x=P, xt=0, rows=4, cols=64, ldx=64, f=F4, rounding=0, rule=0, group=32, codes=P, ldc=8, scales=P, lds=2, xq=None, qt=0, ldq=0):
    return lib.esb_project_groups(x, xt, rows, cols, ldx, f, rounding, rule, group, codes, ldc, scales, lds, xq, qt, ldq, None)


@pytest.mark.parametrize("want,kw", [
    (UNS, dict(f=esb.esb_format(9, 2, 1))), (UNS, dict(f=esb.esb_format(4, 4, 1))), (UNS, dict(f=esb.Fmt(5, 2).c())),
    (UNS, dict(f=esb.Fmt(2, 0).c())), (UNS, dict(group=16)), (UNS, dict(group=-32)), (UNS, dict(group=33)),
    (INV, dict(xt=3)), (INV, dict(xt=-1)), (INV, dict(rounding=2)), (INV, dict(rule=2)), (INV, dict(rows=-1)), (INV, dict(cols=-1)),
    (INV, dict(ldx=63)), (INV, dict(ldc=7)), (INV, dict(lds=1)), (INV, dict(x=None)), (INV, dict(codes=None)), (INV, dict(scales=None)),
    (INV, dict(xq=P, qt=5, ldq=64)), (INV, dict(xq=P, ldq=63)), (ALN, dict(x=ODD)), (ALN, dict(codes=ODD)), (ALN, dict(scales=ODD)),
    (ALN, dict(xq=ODD, qt=1, ldq=64)), (0, dict(rows=0, x=None)), (0, dict(cols=0, ldx=0)),
])
def test_project_groups_refuses(lib, want, kw):
    assert project(lib, **kw) == want


def coded(codes=P, ld=8, scales=P, lds=2, group=32, fmt=F4):
    return esb.esb_coded(codes, ld, scales, lds, group, fmt)


def matvec(lib, M=2, N=8, K=64, x=P, xt=0, ldx=64, xc=None, w=None, bias=None, y=P, yt=0, ldy=8, no_w=False):
    w = coded() if w is None else w
    return lib.esb_matvec_groups(M, N, K, x, xt, ldx, ctypes.byref(xc) if xc else None, None if no_w else ctypes.byref(w), bias, y, yt,
                                 ldy, None)


X8 = dict(ld=16, lds=1, group=0, fmt=F8)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(no_w=True)), (INV, dict(xt=4)), (INV, dict(yt=3)), (INV, dict(xt=3)), (INV, dict(M=-1)), (INV, dict(N=-1)), (INV, dict(K=-1)),
    (INV, dict(K=0)), (INV, dict(ldx=63)), (INV, dict(ldy=7)), (INV, dict(x=None)), (INV, dict(y=None)),
    (INV, dict(w=coded(codes=None))), (INV, dict(w=coded(scales=None))), (INV, dict(w=coded(ld=4))), (INV, dict(w=coded(lds=1))),
    (UNS, dict(w=coded(fmt=F8))), (UNS, dict(w=coded(fmt=esb.esb_format(4, 4, 1)))), (UNS, dict(w=coded(group=48))),
    (UNS, dict(w=coded(group=-32))), (RNG, dict(K=1 << 18, ldx=1 << 18, w=coded(ld=1 << 15, lds=1 << 13))),
    (ALN, dict(w=coded(codes=ctypes.c_void_p(264)))), (ALN, dict(w=coded(ld=9))), (ALN, dict(w=coded(scales=ODD))), (ALN, dict(x=ODD)),
    (ALN, dict(y=ODD)), (ALN, dict(bias=ODD)),
    (UNS, dict(xt=3, xc=coded(ld=16, lds=1, group=0, fmt=F4))), (UNS, dict(xt=3, xc=coded(ld=16, lds=1, group=0, fmt=esb.Fmt(8, 1).c()))),
    (UNS, dict(xt=3, xc=coded(ld=16, lds=2, group=48, fmt=F8))), (UNS, dict(xt=3, xc=coded(ld=16, lds=2, group=32, fmt=F8), w=coded(group=0))),
    (INV, dict(xt=3, xc=coded(codes=None, **X8))), (INV, dict(xt=3, xc=coded(scales=None, **X8))),
    (INV, dict(xt=3, xc=coded(**{**X8, "ld": 15}))), (INV, dict(xt=3, xc=coded(**{**X8, "lds": 0}))),
    (ALN, dict(xt=3, xc=coded(codes=ODD, **X8))), (0, dict(M=0)), (0, dict(N=0, ldy=0)),
])
def test_matvec_groups_refuses(lib, want, kw):
    assert matvec(lib, **kw) == want


def norm(lib, rows=2, cols=64, null=False, **kw):
    a = esb.esb_norm(x=P, ldx=64, residual=P, ldr=64, weight=P, h=P, ldh=64, y=P, ldy=64, rstd=P, codes=P, ldc=16, scales=P, lds=2,
                     yq=P, ldq=64, group=32, fmt=F8, rounding=0, x_type=0, w_type=0, y_type=0, eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return lib.esb_rmsnorm(rows, cols, None if null else ctypes.byref(a), None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(rows=-1)), (INV, dict(cols=-1)), (INV, dict(eps=-1.0)), (INV, dict(eps=float("nan"))),
    (INV, dict(eps=float("inf"))), (INV, dict(x_type=3)), (INV, dict(w_type=7)), (INV, dict(y_type=3)), (INV, dict(x=None)),
    (INV, dict(ldx=63)), (INV, dict(ldr=63)), (INV, dict(ldh=63)), (INV, dict(ldy=63)), (INV, dict(ldq=63)), (INV, dict(ldc=15)),
    (INV, dict(lds=1)), (INV, dict(scales=None)), (INV, dict(rounding=2)), (INV, dict(codes=None)),
    (UNS, dict(fmt=F4)), (UNS, dict(fmt=esb.esb_format(8, 8, 1))), (UNS, dict(group=24)), (UNS, dict(group=-64)),
    (ALN, dict(x=257)), (ALN, dict(residual=258, x_type=0)), (ALN, dict(weight=257)), (ALN, dict(h=257)), (ALN, dict(y=257)),
    (ALN, dict(yq=257)), (ALN, dict(rstd=257)), (ALN, dict(codes=257)), (ALN, dict(scales=257)),
    (0, dict(rows=0)), (0, dict(cols=0)),
])
def test_rmsnorm_refuses(lib, want, kw):
    assert norm(lib, **kw) == want


def norm_grad(lib, rows=2, cols=64, null=False, ws=P, nb=1 << 20, **kw):
    a = esb.esb_norm_grad(dy=P, ldg=64, h=P, ldh=64, dh=P, lddh=64, weight=P, rstd=P, dx=P, lddx=64, dweight=P, x_type=0, w_type=0, g_type=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return lib.esb_rmsnorm_backward(rows, cols, None if null else ctypes.byref(a), ws, nb, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(rows=-1)), (INV, dict(cols=-1)), (INV, dict(x_type=3)), (INV, dict(g_type=3)), (INV, dict(w_type=-1)),
    (INV, dict(dy=None)), (INV, dict(h=None)), (INV, dict(rstd=None)), (INV, dict(dx=None)), (INV, dict(ldg=63)), (INV, dict(ldh=63)),
    (INV, dict(lddh=63)), (INV, dict(lddx=63)), (INV, dict(ws=None)), (INV, dict(nb=4)), (ALN, dict(ws=ctypes.c_void_p(264))),
    (ALN, dict(dy=257)), (ALN, dict(h=257)), (ALN, dict(dh=257)), (ALN, dict(dx=257)), (ALN, dict(weight=257)), (ALN, dict(rstd=257)),
    (ALN, dict(dweight=257)), (0, dict(rows=0, dweight=None)), (0, dict(cols=0)),
])
def test_rmsnorm_backward_refuses(lib, want, kw):
    assert norm_grad(lib, **kw) == want


def logprobs(lib, x=P, xt=0, rows=2, cols=64, ldx=64, ids=P, top=2, logp=P, ent=P, lse=P, tl=P, ti=P):
    return lib.esb_logprobs(x, xt, rows, cols, ldx, ids, top, logp, ent, lse, tl, ti, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(xt=3)), (INV, dict(rows=-1)), (INV, dict(cols=-1)), (INV, dict(top=-1)), (INV, dict(ids=None)), (INV, dict(x=None)),
    (INV, dict(cols=0)), (INV, dict(ldx=63)), (INV, dict(tl=None)), (INV, dict(ti=None)), (RNG, dict(top=33)),
    (RNG, dict(cols=1 << 31, ldx=1 << 31)), (ALN, dict(x=ODD)), (ALN, dict(ids=ctypes.c_void_p(260))), (ALN, dict(ti=ctypes.c_void_p(260))),
    (ALN, dict(logp=ODD)), (ALN, dict(ent=ODD)), (ALN, dict(lse=ODD)), (ALN, dict(tl=ODD)), (0, dict(rows=0)),
])
def test_logprobs_refuses(lib, want, kw):
    assert logprobs(lib, **kw) == want


def logprobs_grad(lib, x=P, xt=0, rows=2, cols=64, ldx=64, ids=P, lse=P, ent=P, dl=P, de=P, dx=P, lddx=64):
    return lib.esb_logprobs_backward(x, xt, rows, cols, ldx, ids, lse, ent, dl, de, dx, lddx, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(xt=3)), (INV, dict(rows=-1)), (INV, dict(cols=-1)), (INV, dict(ids=None)), (INV, dict(ent=None)), (INV, dict(x=None)),
    (INV, dict(lse=None)), (INV, dict(dx=None)), (INV, dict(ldx=63)), (INV, dict(lddx=63)), (RNG, dict(cols=1 << 31, ldx=1 << 31)),
    (ALN, dict(x=ODD)), (ALN, dict(dx=ODD)), (ALN, dict(ids=ctypes.c_void_p(260))), (ALN, dict(lse=ODD)), (ALN, dict(dl=ODD)),
    (0, dict(rows=0)), (0, dict(cols=0)),
])
def test_logprobs_backward_refuses(lib, want, kw):
    assert logprobs_grad(lib, **kw) == want


def test_binding_refuses_host_tensors_and_shapes(lib):
    x = torch.zeros(4, 64)
    for call in (lambda: esb.esb_project_groups(x, esb.Fmt(4, 2)), lambda: esb.esb_rmsnorm(x, None), lambda: esb.esb_logprobs(x),
                 lambda: esb.esb_project_groups(x.double(), esb.Fmt(4, 2)),
                 lambda: esb.esb_matvec_groups(x, esb.Coded(torch.zeros((4, 8), dtype=torch.int32), torch.zeros((4, 1)), esb.Fmt(4, 2), 64)),
                 lambda: esb.esb_rmsnorm_backward(x, x, None, torch.zeros(4)),
                 lambda: esb.esb_logprobs_backward(x, None, torch.zeros(4))):
        with pytest.raises(ValueError):
            call()
