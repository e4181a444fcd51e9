"""A decoder's attention at its edges: many queries on one head of the cache,
lengths far past the page table."""
import pytest
import torch

from paper_2109_03513_gb300 import esb
from test_gpu_attention import check_attention, i32, ints, make_cache, tables
from test_gpu_lm import TYPES, rand

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
