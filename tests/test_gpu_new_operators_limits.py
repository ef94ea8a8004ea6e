"""Arguments at the ends of their ranges for the operators on new tokens and on the cache's pages."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_new_tokens import Cache, queries, run_tree, run_window, sent, workspace
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


@pytest.mark.parametrize("max_pages", [1, 7, 300, 20000])
def test_ranges_of_pages_far_outside_the_row(max_pages):
    """First and last pages of any 32-bit value: what lies in the row is given back, nothing else is touched."""
    import paper_2502_02770_amd as T
    most, least = 2**31 - 1, -2**31
    ranges = [(most, 0), (most, most), (least, least), (most, least), (least, 0), (max_pages, most), (most - 5, most), (max_pages + 1, 0),
              (0, least), (least, 2), (max_pages - 1, most), (0, 0)]
    n = len(ranges)
    # rows of others on both sides of every row: the whole table is checked
    table = np.arange(n * max_pages, dtype=np.int32).reshape(n, max_pages)
    c = cache_of(table, [0] * n, n * max_pages, 1, 1, fill=False)
    p = T.PagePool(c)
    p.free(i32([r[0] for r in ranges]), i32([r[1] for r in ranges]))
    for b, (lo, hi) in enumerate(ranges):
        table[b, max(lo, 0):max(0, min(hi, max_pages))] = -1
    assert np.array_equal(c.page_table.cpu().numpy(), table) and int(p.status) == 0
    count = np.ones(n * max_pages, dtype=np.int32)
    count[np.setdiff1d(np.arange(n * max_pages), table[table >= 0])] = 0
    assert np.array_equal(p.ref_count.cpu().numpy(), count)


def test_masks_on_the_device_and_in_a_graph():
    from paper_2502_02770_amd.cache import tree_mask_of_parents
    rng = np.random.default_rng(0)
    ps = [i32(np.floor(rng.random((5, 130)) * (np.arange(130) + 1)) - 1) for _ in range(2)]
    ps[1][2, 7:40] = 2**31 - 1                                     # no tokens of the draft
    want = [tree_mask_of_parents(p.cpu()).cuda() for p in ps]
    at = ps[0].clone()
    assert torch.equal(tree_mask_of_parents(at), want[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = tree_mask_of_parents(at)
    for turn in range(4):
        at.copy_(ps[turn % 2])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[turn % 2])


@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 2)])
@pytest.mark.parametrize("n,new", [(70, 1), (70, 9), (3000, 1), (3000, 9), (3000, 40)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_not_finite_show_it_in_lse_too(n, new, hq, hkv, bad):
    """-inf stands for rows that see nothing; lists taken whole and cut ones."""
    import paper_2502_02770_amd as T
    c = Cache([n], hq, hkv, seed=n)
    q = queries(new, hq, 1)
    q[new // 2, 3] = bad                                           # inf: scores of either infinity
    mask = np.full((new, -(-new // 32)), -1, dtype=np.int32)
    calls = (lambda o, l: T.twilight_window_attention(c.kv, q, None, None, new, 2**31 - 1, 0, o, l, workspace(c.kv, new)),
             lambda o, l: T.twilight_tree_attention(c.kv, q, None, None, new, i32(mask), mask.shape[1], o, l, workspace(c.kv, new)))
    for call in calls:
        out, lse = sent(q, hq)
        call(out, lse)
        mine = torch.zeros(new, hq, dtype=torch.bool, device="cuda")
        mine[new // 2, 3] = True
        assert torch.isnan(out[mine]).all() and torch.isnan(lse[mine]).all()
        assert torch.isfinite(out[~mine]).all() and torch.isfinite(lse[~mine]).all()
