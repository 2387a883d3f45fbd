"""spec_page_select reports ids that are no pages for every sequence whose pages it lists, those that read all they have too."""
import numpy as np
import pytest

from paper_2504_00030_b200 import binding as sv
from tests.longctx import config
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths", [[100, 3000], [100, 140]], ids=["beside one that is scored", "no scores at all"])
@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_sequences_that_read_all_their_pages(lengths, bad):
    cfg = config("pt", 2, 4, 2, 128, 27)
    table, cu, q, bounds, scales = setup(cfg, lengths, [2, 1], 2, 1)
    call = lambda t: select_gpu(cfg, q, bounds, scales, t, lengths, [2, 1], cu, 2, 10, 1, 1)  # noqa: E731
    table[0, 7:] = bad                                    # behind its seven pages: not looked at
    pl, rm, n, status = call(table)
    assert status == 0
    for page in (0, 3, 6):
        broken = table.copy()
        broken[0, page] = bad
        p2, r2, n2, status = call(broken)
        assert status == sv.SV_DEV_BAD_PAGE
        for a, b in ((pl, p2), (rm, r2), (n, n2)):        # and the lists are what they are
            np.testing.assert_array_equal(a, b)
        assert n[0].tolist() == [7, 7] and pl[0, 0, :7].tolist() == list(range(7))


def test_many_pages_none_left_out():
    """More pages than a block has threads."""
    cfg = config("pt", 1, 2, 1, 64, 28)
    table, cu, q, bounds, scales = setup(cfg, [16000], [0], 0, 1)
    assert select_gpu(cfg, q, bounds, scales, table, [16000], [0], cu, 0, 1000, 1, 1)[3] == 0
    for page in (999, 640, 31):
        broken = table.copy()
        broken[0, page] = len(scales)
        assert select_gpu(cfg, q, bounds, scales, broken, [16000], [0], cu, 0, 1000, 1, 1)[3] == sv.SV_DEV_BAD_PAGE
