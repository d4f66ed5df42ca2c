"""The paged key/value cache on the GPU at the ends of its types' ranges."""
import numpy as np
import pytest
import torch

from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, Pool, dev

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ select

@pytest.mark.parametrize("n_pages", [8, 70])
def test_scores_below_the_range_rank_above_nan(n_pages):
    """Scores of finite queries and keys past float32's range on the negative
    side are numbers, and NaN ranks below every number."""
    say(f"paged select, scores below the range, {n_pages} pages")
    pool = Pool("int8", [16 * n_pages], 1, 64, 16, with_bounds=True, width_extra=0)
    pool.db[:] = -3
    pool.dbe[:] = 127 + 100
    pool.dbe[0, torch.from_numpy(pool.table[0, [0, 3]].astype(np.int64)).cuda()] = 255
    q = dev(np.full((1, 64), 2.0 ** 100), torch.bfloat16)
    numbers = [p for p in range(n_pages) if p not in (0, 3)]
    for k, want in ((2, numbers[:2]), (n_pages - 2, numbers), (n_pages - 1, [0] + numbers)):
        pages = torch.full((1, 1, k), -5, dtype=torch.int32, device="cuda")
        binding.paged_select(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 1, q, 64, None, 1, 1, DT["bf16"], k,
                             pages)
        assert pages[0, 0].tolist() == want
