"""spec_page_select where the chosen bits of a block's rows take more and more memory: shared memory that a kernel has to ask
for, and the workspace.  Both go by gamma_max and max_seq_len; the sequences may be short."""
import pytest

from tests.longctx import config
from tests.test_gpu_page_select import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gmax,most", [(22, 262144), (31, 190000), (16, 350000), (63, 92000)])
def test_just_under_what_a_kernel_has_without_asking(gmax, most):
    """46 to 48 KB beside the kernel's own arrays."""
    check(config("pb", 2, 4, 2, 64, 24), [1500, 200], [gmax, 3], gmax, 12, 1, 2, most=most)


@pytest.mark.parametrize("gmax,most", [(63, 150000), (31, 300000), (63, 260000), (40, 600000)])
def test_bits_in_much_shared_memory_and_in_the_workspace(gmax, most):
    """75 KB in shared memory; 130 and 196 KB for each sequence and kv head in the workspace."""
    check(config("pb", 3, 4, 2, 64, 25), [5000, 90, 1700], [gmax, 5, gmax], gmax, 20, 1, 2, most=most)
    check(config("pb", 2, 2, 2, 128, 26), [3001, 64 + gmax], [gmax, gmax], gmax, 9, 0, 1, few=True, most=most)
