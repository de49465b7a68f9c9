"""Page calls at the sizes where their counting changes: caches of 4096 pages and a few more or fewer, many reservations in a small one."""
import pytest

import test_gpu_kv4_pages as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages,seqs,cols,page_bytes,seed", [(1000, 150, 8, 64, 6), (4095, 90, 40, 32, 7), (4096, 140, 60, 16, 8), (4097, 200, 30, 16, 9)])
def test_sizes(pages, seqs, cols, page_bytes, seed):
    base.test_a_scheduler_s_day(pages, seqs, cols, page_bytes, seed)
