"""The binding of the language-model operators refuses code tensors whose rows
would be read or written outside of them (host checks; runs without a GPU)."""
import pytest
import torch

from paper_2109_03513_gb300 import esb


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device: every call here is refused before anything reads it."""
    is_cuda = True


def dev(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def lib():
        raise AssertionError("the call was not refused")
    monkeypatch.setattr(esb, "lib", lib)


def test_codes_are_written_into_whole_rows_only():
    # every word of a row's stride is written: a view of some columns would have its neighbours overwritten
    wide = dev(4, 64, dtype=torch.int32)
    x = dev(4, 64)
    for codes in (wide[:, :8], wide[:, 56:], wide[:1].expand(4, 64), wide[::2], dev(3, 16, dtype=torch.int32)):
        with pytest.raises(ValueError):
            esb.esb_project_groups(x, esb.Fmt(4, 2), 32, codes=codes)
        with pytest.raises(ValueError):
            esb.esb_rmsnorm(x, None, fmt=esb.Fmt(8, 6), group=32, codes=codes)


def test_codes_hold_the_columns_that_are_read():
    wide, scales, x = dev(4, 64, dtype=torch.int32), dev(4, 2), dev(1, 64)
    for codes in (wide[:, :4], wide[:, 60:], wide[:, :7]):
        with pytest.raises(ValueError):
            esb.esb_matvec_groups(x, esb.Coded(codes, scales, esb.Fmt(4, 2), 64, 32))
    w = esb.Coded(wide[:, :8], scales, esb.Fmt(4, 2), 64, 32)
    with pytest.raises(ValueError):
        esb.esb_matvec_groups(esb.Coded(wide[:, :15], dev(4, 1), esb.Fmt(8, 6), 64), w)
    with pytest.raises(AssertionError):      # these hold them
        esb.esb_matvec_groups(esb.Coded(wide[:, :16], dev(4, 1), esb.Fmt(8, 6), 64), w, y=dev(4, 4))
