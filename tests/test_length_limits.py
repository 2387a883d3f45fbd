"""Bounds of the sequence lengths up to the largest 32-bit number: refused on the host where the block table does not hold them."""
import ctypes as C

import pytest

from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import build as svbuild
from tests.test_long_context_refusals import P, attn, made, pool

LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    svbuild.build()
    return sv.load()


@pytest.mark.parametrize("longest", [LAST, LAST - 14, LAST - 15, 161])
def test_table_rows_that_are_too_short(lib, longest):
    pl = pool()
    at = attn(pl, max_seq_len=longest)                     # ten pages a row
    assert lib.spec_verify_attn(C.byref(at), P, 1 << 40, None) == sv.SV_EINVAL
    lists = made(sv.AttnPagesParams, dict(attn=at, page_list=P, row_mask=P, n_list=P, list_stride=10))
    assert lib.spec_verify_attn_pages(C.byref(lists), P, 1 << 40, None) == sv.SV_EINVAL
    behind = made(sv.AttnPrefixParams, dict(attn=at, group=P, prefix_len=P, n_groups=2))
    assert lib.spec_verify_attn_prefix(C.byref(behind), P, 1 << 40, None) == sv.SV_EINVAL
    select = made(sv.PageSelectParams, dict(q=P, bounds=P, scales=P, n_pages=100, block_table=P, block_table_stride=10, seq_len=P, gamma=P, cu_q=P, batch=3,
                                            gamma_max=4, hq=8, hkv=2, head_dim=128, max_seq_len=longest, n_select=4, n_first=1, n_last=2, page_list=P,
                                            row_mask=P, n_list=P, list_stride=20))
    assert lib.spec_page_select(C.byref(select), P, 1 << 40, None) == sv.SV_EINVAL


def test_lengths_whose_last_tile_no_int_numbers(lib):
    """The attentions over parts of the cache take lengths up to 2^31 - 65."""
    pl = pool()
    for longest, want in ((LAST, sv.SV_EUNSUPPORTED), (LAST - 63, sv.SV_EUNSUPPORTED), (LAST - 64, sv.SV_EWORKSPACE)):
        at = attn(pl, max_seq_len=longest, block_table_stride=(longest + 15) // 16, batch=1)
        lists = made(sv.AttnPagesParams, dict(attn=at, page_list=P, row_mask=P, n_list=P, list_stride=10))
        assert lib.spec_verify_attn_pages(C.byref(lists), P, 0, None) == want
        behind = made(sv.AttnPrefixParams, dict(attn=at, group=P, prefix_len=P, n_groups=1))
        assert lib.spec_verify_attn_prefix(C.byref(behind), P, 0, None) == want
