"""Attention over a cache in 4 bits where a KV head has several row blocks: windows that meet a tile's border."""
import pytest

from tests.kv4_util import Cache4
from tests.test_gpu_kv4 import attend

pytestmark = pytest.mark.gpu


# A row block's list may have a tile more than that of the sequence's last tokens, as it lies differently against the pages.
@pytest.mark.parametrize("hq,hkv,lens,new,window,sinks", [
    (32, 8, [4096], 12, 505, 0),                 # blocks of 32 rows: the first has 3 tiles, that of the last 8 tokens 2
    (16, 8, [17087], 171, 1024, 0),              # of 128 rows: 18 and 17
    (32, 32, [24639], 391, 2048, 0),             # 35 and 34
    (32, 8, [4096], 257, 2017, 0),               # 33 and 32
    (32, 8, [3654] * 6, 85, 2244, 16),
    (64, 8, [8059], 7, 1255, 4),
])
def test_blocks_that_see_a_page_more_than_the_last_one(hq, hkv, lens, new, window, sinks):
    attend(Cache4(lens, hq, hkv, seed=new), [new] * len(lens), new, window, sinks, seed=window)


@pytest.mark.parametrize("sinks", [0, 3, 40])
@pytest.mark.parametrize("edge", [-9, -8, -7, -4, -1, 0, 1, 2])
@pytest.mark.parametrize("hq,hkv,new", [(32, 8, 13), (16, 2, 9), (8, 8, 61), (32, 8, 99), (16, 2, 50), (8, 8, 267)])
def test_windows_at_the_border_of_a_tile(hq, hkv, new, edge, sinks):
    """Cut lists of both kernels, windows of whole tiles and some tokens less or more."""
    lens = [3000 + 7 * new, 2741]
    attend(Cache4(lens, hq, hkv, seed=new), [new, new - 1], new, 1024 + edge, sinks, seed=new + edge)
