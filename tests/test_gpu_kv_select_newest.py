"""Which rows count as the newest ones of a sequence."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_kv_evict import row_numbers

pytestmark = pytest.mark.gpu


def test_the_newest_of_none_at_the_end_of_the_positions():
    """`recent` = 0 protects nothing, also where a position is the largest that there is."""
    s = R.Setup([60], 1, 16, 16, 16, seed=1)
    cache = s.cache()
    marks, row = B.KVMarks(cache), row_numbers(s, 0, 0, 60).cuda()
    marks.pos.view(-1)[row] = 2 ** 31 - 1
    marks.mass.view(-1)[row] = torch.arange(60, dtype=torch.float32, device="cuda")
    source, _ = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 20, 0)
    cache.check()
    assert source[0, 0].tolist() == list(range(40, 60))
