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
