"""Forms of the attention kernels that only some sizes reach, each by a case made for its rule."""
import pytest

import kv_cases as K
from test_gpu_kv import check_attend, check_blocks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_amd import kv
    return kv


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group,new", [(11, 1), (12, 1), (16, 1), (3, 5), (17, 1), (4, 8), (6, 5)])
def test_scores_of_one_long_chunk(kv, dtype, group, new):
    """One block a sequence and kv head, 1,024 entries: the scores of 11 rows and more do not fit LDS and go to memory
    as they come."""
    check_attend(kv, K.Case(dtype, 64, 16, 2, group, (1000, 37), (new, 1), missing=[(0, 5), (0, 62)], seed=group))


@pytest.mark.parametrize("dim,group,new", [(64, 4, 2), (64, 4, 8), (128, 8, 1), (128, 5, 3)])
def test_scores_of_long_chunks(kv, dim, group, new):
    """80 pairs under a bound of 100,000 entries: chunks of 2,048, their scores too large for LDS, some sequences with
    several of them and an end inside a run of 64."""
    lens = [1 + (i * 37) % 300 for i in range(36)] + [2048, 2049, 4133, 2090]
    c = K.Case("bf16", dim, 32, 2, group, lens, [min(n, new) for n in lens], max_pages=4000, missing=[(38, 64), (39, 1)],
               seed=dim + group)
    check_attend(kv, c, max_len=100000)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,new", [((200, 33), (1, 1)), ((200, 64), (2, 1)), ((777, 90), (1, 2)), ((1290,), (1,))])
@pytest.mark.parametrize("group", [9, 16, 17, 24, 32])
def test_scores_of_two_row_tiles_of_wide_heads(kv, dtype, lens, new, group):
    """17 to 32 rows of 256 dimensions: the launch that takes the most registers and LDS, in one split and in several, a
    last run of less than 64 entries, and pages that are not there."""
    new = [min(n, 32 // group) for n in new]
    check_attend(kv, K.Case(dtype, 256, 16, 1, group, lens, new, missing=[(0, 2), (0, 12)], seed=group))


@pytest.mark.parametrize("dtype,dim,page", [("bf16", 64, 16), ("fp16", 64, 64), ("bf16", 256, 32), ("fp16", 256, 16),
                                            ("bf16", 128, 64), ("fp16", 128, 32)])
@pytest.mark.parametrize("group", [17, 32, 33, 50])
@pytest.mark.parametrize("n_sel", [3, 30])
def test_blocks_of_large_groups(kv, dtype, dim, page, group, n_sel):
    """Sparse attention of more than 16 query heads a kv head: two row tiles a wavefront, and blocks of them."""
    c = K.Case(dtype, dim, page, 1, group, (900, 5, 70), (2, 1, 3), missing=[(0, 3)], seed=group)
    check_blocks(kv, c, n_sel, 1, 2)
