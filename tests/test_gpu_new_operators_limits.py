"""Arguments at the ends of their ranges for the operators on new tokens and on the cache's pages."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_pages import cache_of, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(2**31 - 1, 0), (2**32, 4), (2**40, 0), (2**63 - 1, 3), (40, 2**36)])
def test_windows_and_sinks_without_limit_keep_every_page(window, sinks):
    import paper_2502_02770_amd as T
    c = cache_of(np.arange(2 * 63).reshape(2, 63), [1000, 64], 130, fill=False)
    p = T.PagePool(c)
    table, count = c.page_table.clone(), p.ref_count.clone()
    p.free_behind(window, sinks)
    assert torch.equal(c.page_table, table) and torch.equal(p.ref_count, count) and int(p.status) == 0
