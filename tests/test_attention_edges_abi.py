"""Refusals at the edges of a decoder's attention: host-side validation of the C
ABI (no device work; runs without a GPU)."""
import pytest

from test_attention_abi import INV, append, attend, grad, lib, norm, turn


@pytest.mark.parametrize("call", [norm, grad, append, attend])
def test_a_table_of_no_rows_is_refused(lib, call):
    # kernels read row 0 for a position that the table lacks, and drop it
    none = turn(positions=0)
    kw = dict(rotation=none) if call in (norm, grad) else dict(r=none)
    assert call(lib, **kw) == INV
    assert call(lib, tokens=0, **dict(kw, **(dict(q=dict(dweight=None), k=dict(dweight=None)) if call is grad else {}))) == 0
