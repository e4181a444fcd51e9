"""The binding of a decoder's attention refuses tensors of another device than
the current one, whichever of a call they are (host checks; runs without a GPU)."""
import pytest
import torch

from paper_2109_03513_gb300 import esb

I32, I64, F32 = torch.int32, torch.int64, torch.float32


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device: nothing here gets as far as reading it."""
    is_cuda = True
    where = 0

    def get_device(self):
        return self.where


class Elsewhere(OnDevice):
    where = 1


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def device_0(monkeypatch):
    def lib():
        raise Reached
    monkeypatch.setattr(esb, "lib", lib)
    monkeypatch.setattr(esb, "_current_device", lambda: 0)
    monkeypatch.setattr(esb, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)


def t(*shape, dtype=F32):
    return lambda kind: torch.zeros(shape, dtype=dtype).as_subclass(kind)


CACHE = dict(k_codes=t(4, 2, 16, 8, dtype=I32), k_scales=t(4, 2, 16), v_codes=t(4, 2, 16, 8, dtype=I32), v_scales=t(4, 2, 16))


def cache(m):
    return esb.KvCache(m["k_codes"], m["k_scales"], m["v_codes"], m["v_scales"], 64, esb.Fmt(4, 2), esb.Fmt(4, 2))


def append(m):
    esb.esb_cache_append(cache(m), m["k"], m["v"], m["slots"], rotation=esb.Rotation(m["table"]), positions=m["positions"], kq=m["kq"], vq=m["vq"])


def attend(m):
    esb.esb_cache_attention(m["q"], cache(m), m["lens"], m["pages"], starts=m["starts"], rotation=esb.Rotation(m["table"]), out=m["out"], workspace=m["workspace"])


def norm(m):
    esb.esb_headnorm(m["q"], m["k"], 64, m["qw"], m["kw"], rotation=esb.Rotation(m["table"]), positions=m["positions"], qy=m["qy"], ky=m["ky"])


def grad(m):
    esb.esb_headnorm_backward(m["gq"], m["gk"], m["q"], m["k"], 64, m["qw"], m["kw"], m["qr"], m["kr"], rotation=esb.Rotation(m["table"]),
                              positions=m["positions"], dq=m["dq"], dk=m["dk"], workspace=m["workspace"])


x, pos, table, w, space = t(3, 128), t(3, dtype=I64), t(10, 64), t(64), t(1 << 12, dtype=torch.uint8)
CALLS = [
    (append, dict(CACHE, k=x, v=x, slots=pos, positions=pos, table=table, kq=x, vq=x)),
    (attend, dict(CACHE, q=x, lens=t(3, dtype=I32), pages=t(3, 2, dtype=I32), starts=t(4, dtype=I32), table=table, out=x, workspace=space)),
    (norm, dict(q=x, k=x, qw=w, kw=w, positions=pos, table=table, qy=x, ky=x)),
    (grad, dict(gq=x, gk=x, q=x, k=x, qw=w, kw=w, qr=t(3, 2), kr=t(3, 2), positions=pos, table=table, dq=x, dk=x, workspace=space)),
]


@pytest.mark.parametrize("call,makers,other", [(c, m, name) for c, m in CALLS for name in [None, *m]])
def test_every_tensor_is_on_the_current_device(call, makers, other):
    with pytest.raises(Reached if other is None else ValueError):
        call({name: make(Elsewhere if name == other else OnDevice) for name, make in makers.items()})
