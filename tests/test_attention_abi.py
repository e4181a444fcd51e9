"""Refusals of a decoder's attention: host-side validation of the C ABI and of
the binding (no device work; runs without a GPU)."""
import ctypes

import pytest
import torch

from paper_2109_03513_gb300 import esb

P, ODD = 256, 257                   # an aligned address that nothing reads: every call here is refused, or has nothing to do
INV, UNS, RNG, ALN = esb.ESB_ERR_INVALID_ARG, esb.ESB_ERR_UNSUPPORTED, esb.ESB_ERR_RANGE, esb.ESB_ERR_ALIGN
F4 = esb.Fmt(4, 2).c()


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__
    __graft_entry__.build()
    return esb.lib()


def turn(table=P, positions=10, ld=64, dim=64, interleaved=0):
    return esb.esb_rotation(table, positions, ld, dim, interleaved)


def fill(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


# ------------------------------------------------------------- norms of heads

def norm(lib, tokens=3, null=False, q=None, k=None, **kw):
    a = esb.esb_head_norm(positions=P, rotation=turn(), head_dim=64, x_type=0, w_type=0, eps=1e-6)
    for part, change in ((a.part[0], q), (a.part[1], k)):
        fill(part, dict(dict(x=P, ldx=128, y=P, ldy=128, weight=P, rstd=P, heads=2), **(change or {})))
    return lib.esb_headnorm(tokens, None if null else ctypes.byref(fill(a, kw)), None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(tokens=-1)), (RNG, dict(tokens=1 << 31)), (INV, dict(eps=-1.0)), (INV, dict(eps=float("nan"))),
    (INV, dict(x_type=3)), (INV, dict(w_type=7)), (UNS, dict(head_dim=60)), (UNS, dict(head_dim=0)), (UNS, dict(head_dim=264)),
    (UNS, dict(rotation=turn(dim=63))), (UNS, dict(rotation=turn(dim=66))), (UNS, dict(rotation=turn(dim=-2))), (INV, dict(rotation=turn(ld=63))),
    (INV, dict(rotation=turn(table=None))), (INV, dict(positions=None)), (ALN, dict(rotation=turn(table=ODD))), (ALN, dict(positions=260)),
    (INV, dict(q=dict(heads=-1))), (RNG, dict(k=dict(heads=1 << 23))), (INV, dict(q=dict(x=None))), (INV, dict(k=dict(y=None))),
    (INV, dict(q=dict(ldx=127))), (INV, dict(k=dict(ldy=127))), (ALN, dict(q=dict(x=ODD))), (ALN, dict(k=dict(y=ODD))),
    (ALN, dict(q=dict(weight=ODD))), (ALN, dict(k=dict(rstd=ODD))), (0, dict(tokens=0)), (0, dict(q=dict(heads=0), k=dict(heads=0))),
    (0, dict(tokens=0, positions=None)),
])
def test_headnorm_refuses(lib, want, kw):
    assert norm(lib, **kw) == want


def grad(lib, tokens=3, null=False, ws=P, nb=1 << 30, q=None, k=None, **kw):
    a = esb.esb_head_norm_grad(positions=P, rotation=turn(), head_dim=64, x_type=0, w_type=0)
    for part, change in ((a.part[0], q), (a.part[1], k)):
        fill(part, dict(dict(dy=P, ldg=128, x=P, ldx=128, rstd=P, weight=P, dx=P, lddx=128, dweight=P, heads=2), **(change or {})))
    return lib.esb_headnorm_backward(tokens, None if null else ctypes.byref(fill(a, kw)), ws, nb, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(tokens=-1)), (RNG, dict(tokens=1 << 31)), (INV, dict(x_type=3)), (INV, dict(w_type=-1)),
    (UNS, dict(head_dim=4)), (UNS, dict(rotation=turn(dim=65))), (INV, dict(positions=None)), (INV, dict(q=dict(dy=None))),
    (INV, dict(k=dict(x=None))), (INV, dict(q=dict(rstd=None))), (INV, dict(k=dict(dx=None))), (INV, dict(q=dict(ldg=127))),
    (INV, dict(k=dict(ldx=127))), (INV, dict(q=dict(lddx=127))), (INV, dict(ws=None)), (INV, dict(nb=8)), (ALN, dict(ws=264)),
    (ALN, dict(q=dict(dy=ODD))), (ALN, dict(k=dict(x=ODD))), (ALN, dict(q=dict(dx=ODD))), (ALN, dict(k=dict(rstd=ODD))),
    (ALN, dict(q=dict(weight=ODD))), (ALN, dict(k=dict(dweight=ODD))), (INV, dict(q=dict(heads=-3))), (RNG, dict(q=dict(heads=1 << 23))),
    (0, dict(tokens=0, q=dict(dweight=None), k=dict(dweight=None))), (0, dict(q=dict(heads=0, dweight=None), k=dict(heads=0, dweight=None))),
])
def test_headnorm_backward_refuses(lib, want, kw):
    assert grad(lib, **kw) == want


# --------------------------------------------------------------------- cache

def cache(**kw):
    return fill(esb.esb_kv_cache(P, P, P, P, 4, 2 * 16 * 8, 2 * 16, 2, 16, 64, F4, F4), kw)


BAD_CACHES = [
    (UNS, dict(k_fmt=esb.Fmt(8, 6).c())), (UNS, dict(v_fmt=esb.Fmt(4, 2, False).c())), (UNS, dict(k_fmt=esb.esb_format(4, 4, 1))),
    (UNS, dict(head_dim=63)), (UNS, dict(head_dim=264)), (UNS, dict(page_size=0)), (UNS, dict(page_size=24)), (INV, dict(pages=-1)),
    (INV, dict(heads=0)), (RNG, dict(heads=1 << 23)), (RNG, dict(page_size=(1 << 24) + 16)), (RNG, dict(heads=1 << 20, page_size=2048)),
    (RNG, dict(page_ld=1 << 34)), (RNG, dict(page_lds=1 << 32)), (RNG, dict(pages=1 << 40)), (INV, dict(k_codes=None)), (INV, dict(v_codes=None)),
    (INV, dict(k_scales=None)), (INV, dict(v_scales=None)), (INV, dict(page_ld=252)), (INV, dict(page_lds=31)), (ALN, dict(k_codes=264)),
    (ALN, dict(v_codes=ODD)), (ALN, dict(page_ld=258)), (ALN, dict(k_scales=ODD)), (ALN, dict(v_scales=258)),
]


def append(lib, tokens=3, null=False, c=None, r=None, **kw):
    c = cache() if c is None else c
    r = turn() if r is None else r
    a = esb.esb_append(P, P, 128, 128, P, P, ctypes.addressof(r), P, P, 128, 128, 0, 1, 0, 0)
    return lib.esb_cache_append(tokens, ctypes.byref(c), None if null else ctypes.byref(fill(a, kw)), None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(tokens=-1)), (RNG, dict(tokens=1 << 31)), (INV, dict(x_type=3)), (INV, dict(q_type=9)), (INV, dict(rule=2)),
    (INV, dict(rounding=2)), (UNS, dict(r=turn(dim=66))), (INV, dict(positions=None)), (INV, dict(k=None)), (INV, dict(v=None)),
    (INV, dict(slots=None)), (INV, dict(ldk=127)), (INV, dict(ldv=127)), (INV, dict(ldkq=127)), (INV, dict(ldvq=127)), (ALN, dict(k=ODD)),
    (ALN, dict(v=ODD)), (ALN, dict(slots=260)), (ALN, dict(kq=ODD)), (ALN, dict(vq=ODD)), (0, dict(tokens=0)),
] + [(w, dict(c=cache(**k))) for w, k in BAD_CACHES])
def test_append_refuses(lib, want, kw):
    assert append(lib, **kw) == want


def attend(lib, tokens=3, null=False, c=None, r=None, ws=P, nb=1 << 40, **kw):
    c = cache() if c is None else c
    r = turn() if r is None else r
    a = esb.esb_attention(P, 256, P, 256, P, None, P, P, 5, ctypes.addressof(r), 3, 5, 4, 0, 0, 0, 0.125)
    return lib.esb_cache_attention(tokens, ctypes.byref(c), None if null else ctypes.byref(fill(a, kw)), ws, nb, None)


@pytest.mark.parametrize("want,kw", [
    (INV, dict(null=True)), (INV, dict(tokens=-1)), (RNG, dict(tokens=1 << 31)), (INV, dict(seqs=-1)), (INV, dict(max_pages=-1)),
    (INV, dict(window=-1)), (INV, dict(scale=float("nan"))), (INV, dict(scale=float("inf"))), (INV, dict(q_type=3)), (INV, dict(out_type=-1)),
    (UNS, dict(q_heads=3)), (UNS, dict(q_heads=0)), (RNG, dict(q_heads=1 << 24)), (RNG, dict(tokens=1 << 30)), (RNG, dict(max_pages=(1 << 26) + 1)),
    (UNS, dict(r=turn(dim=7))), (INV, dict(r=turn(table=None))), (INV, dict(q=None)), (INV, dict(out=None)), (INV, dict(lens=None)),
    (INV, dict(pages=None)), (INV, dict(ldq=255)), (INV, dict(ldo=255)), (INV, dict(ld_pages=4)), (INV, dict(seqs=2)),
    (ALN, dict(q=ODD)), (ALN, dict(out=ODD)), (ALN, dict(lse=ODD)), (ALN, dict(starts=ODD)), (ALN, dict(lens=ODD)), (ALN, dict(pages=ODD)),
    (INV, dict(ws=None)), (INV, dict(nb=0)), (ALN, dict(ws=264)), (0, dict(tokens=0)), (0, dict(seqs=0)),
] + [(w, dict(c=cache(**k))) for w, k in BAD_CACHES])
def test_attention_refuses(lib, want, kw):
    assert attend(lib, **kw) == want


def test_workspaces(lib):
    for bad in (dict(tokens=0), dict(seqs=0), dict(heads=0), dict(q_heads=3), dict(head_dim=12), dict(q_type=3)):
        kw = dict(dict(tokens=3, seqs=3, q_heads=4, heads=2, head_dim=64, q_type=0), **bad)
        assert lib.esb_cache_attention_workspace_bytes(*kw.values()) == 0
    assert lib.esb_headnorm_backward_workspace_bytes(0, 4, 64) == 0
    assert lib.esb_headnorm_backward_workspace_bytes(5, 4, 60) == 0


# ------------------------------------------------------------------- binding

class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device: every call here is refused before anything reads it."""
    is_cuda = True


def dev(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def no_library(monkeypatch):
    def lib():
        raise AssertionError("the call was not refused")
    monkeypatch.setattr(esb, "lib", lib)


I32, I64 = torch.int32, torch.int64


def kv(**kw):
    c = esb.KvCache(dev(4, 2, 16, 8, dtype=I32), dev(4, 2, 16), dev(4, 2, 16, 8, dtype=I32), dev(4, 2, 16), 64, esb.Fmt(4, 2), esb.Fmt(4, 2))
    return c._replace(**kw)


@pytest.mark.parametrize("kw", [
    dict(k_codes=dev(4, 2, 16, 4, dtype=I32)), dict(k_codes=dev(4, 2, 16, 8)), dict(v_codes=dev(4, 2, 32, 8, dtype=I32)),
    dict(k_scales=dev(4, 2, 16, dtype=torch.float64)), dict(v_scales=dev(4, 2, 8)), dict(head_dim=72), dict(k_codes=dev(4, 2, 16, 16, dtype=I32)[..., :8]),
    dict(k_scales=dev(4, 2, 32)[..., :16]), dict(k_codes=torch.zeros((4, 2, 16, 8), dtype=I32)), dict(v_scales=torch.zeros((4, 2, 16))),
    dict(v_codes=dev(8, 2, 16, 8, dtype=I32)[::2]), dict(v_scales=dev(8, 2, 16)[::2]), dict(k_codes=dev(2, 16, 8, dtype=I32)),
])
def test_binding_refuses_caches(no_library, kw):
    c, x = kv(**kw), dev(3, 128)
    with pytest.raises(ValueError):
        esb.esb_cache_append(c, x, x, dev(3, dtype=I64))
    with pytest.raises(ValueError):
        esb.esb_cache_attention(x, c, dev(3, dtype=I32), dev(3, 2, dtype=I32))


def test_binding_refuses_tensors(no_library):
    c, x, s = kv(), dev(3, 128), dev(3, dtype=I64)
    r = esb.Rotation(dev(10, 64))
    host = torch.zeros(3, 128)
    calls = [
        lambda: esb.esb_cache_append(c, host, x, s), lambda: esb.esb_cache_append(c, x, host, s), lambda: esb.esb_cache_append(c, x, x.half(), s),
        lambda: esb.esb_cache_append(c, dev(3, 64), dev(3, 64), s), lambda: esb.esb_cache_append(c, x, x, s[:2]),
        lambda: esb.esb_cache_append(c, x, x, dev(3, dtype=I32)), lambda: esb.esb_cache_append(c, x, x, s, rotation=r),
        lambda: esb.esb_cache_append(c, x, x, s, rotation=r, positions=s[:1]), lambda: esb.esb_cache_append(c, x, x, s, kq=x[:2]),
        lambda: esb.esb_cache_append(c, x, x, s, kq=x, vq=x.half()), lambda: esb.esb_cache_append(c, x, x, s, kq=x, vq=host),
        lambda: esb.esb_cache_append(c, x, x, s, rotation=esb.Rotation(dev(10, 64).double()), positions=s),
        lambda: esb.esb_cache_append(c, x, x, s, rotation=esb.Rotation(dev(64, 10).t()), positions=s),
        lambda: esb.esb_headnorm(None, None, 64), lambda: esb.esb_headnorm(x, dev(2, 128), 64), lambda: esb.esb_headnorm(x, x.half(), 64),
        lambda: esb.esb_headnorm(x, None, 48), lambda: esb.esb_headnorm(x, None, 0), lambda: esb.esb_headnorm(x, None, 64, dev(63)),
        lambda: esb.esb_headnorm(x, x, 64, dev(64), dev(64).half()), lambda: esb.esb_headnorm(x, None, 64, qy=x.half()),
        lambda: esb.esb_headnorm(x, None, 64, rotation=r), lambda: esb.esb_headnorm(host, None, 64),
        lambda: esb.esb_headnorm_backward(None, None, x, None, 64, None, None, dev(3, 2), None),
        lambda: esb.esb_headnorm_backward(x, None, x, None, 64, None, None, None, None),
        lambda: esb.esb_headnorm_backward(x, None, x, None, 64, None, None, dev(3, 3), None),
        lambda: esb.esb_headnorm_backward(x, None, x, None, 64, None, None, dev(2, 3).t(), None),
        lambda: esb.esb_headnorm_backward(x.half(), None, x, None, 64, None, None, dev(3, 2), None),
        lambda: esb.esb_cache_attention(host, c, dev(3, dtype=I32), dev(3, 2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(3, dtype=I64), dev(3, 2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(3, dtype=I32), dev(2, 2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(3, dtype=I32), dev(2, 3, dtype=I32).t()),
        lambda: esb.esb_cache_attention(x, c, dev(2, dtype=I32), dev(2, 2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(2, dtype=I32), dev(2, 2, dtype=I32), starts=dev(2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(1, 3, dtype=I32), dev(3, 2, dtype=I32)),
        lambda: esb.esb_cache_attention(x, c, dev(3, dtype=I32), dev(3, 2, dtype=I32), out=dev(3, 64)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))


def test_rotation_helper_refuses_and_counts():
    for kw in (dict(dim=3, positions=4), dict(dim=0, positions=4), dict(dim=4, positions=0), dict(dim=4, positions=4, frequencies=[1.0])):
        with pytest.raises(ValueError):
            esb.rotation(device="cpu", **kw)
    r = esb.rotation(4, 3, frequencies=[0.5, 2.0], device="cpu")
    want = torch.tensor([[1, 1, 0, 0]] + [[f(p * w) for f in (torch.cos, torch.sin) for w in (0.5, 2.0)] for p in (torch.tensor(1.0), torch.tensor(2.0))])
    assert r.table.shape == (3, 4) and (r.table - want).abs().max() < 1e-6
