"""Attention over a cache in 4 bits where a KV head has several row blocks: windows that meet a tile's border, and the kernel of 128 rows."""
import math

import pytest
import torch

from tests.kv4_util import Cache4
from tests.test_gpu_kv4 import NONE, attend, check, workspace
from tests.test_gpu_new_tokens import i32, queries, sent

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


WIDE = pytest.mark.parametrize("hq,hkv,new", [(8, 8, 300), (32, 8, 70), (16, 2, 67)])


@WIDE
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 16), (63, 17), (64, 0), (129, 70), (500, 3), (4000, 64), (NONE, 5)])
def test_windows_with_many_rows(hq, hkv, new, window, sinks):
    lens = [40, 513, 1700, 65, 4200]
    attend(Cache4(lens, hq, hkv, seed=window % 1000 + sinks), [min(new, n) for n in lens], new, window, sinks, seed=sinks)


@WIDE
def test_pages_that_are_not_there_with_many_rows(hq, hkv, new):
    c = Cache4([2900, 320, 33], hq, hkv)
    for b, p, v in ((0, 0, -1), (0, 7, 1 << 30), (0, 43, -5), (0, 44, -1), (0, 45, -1), (0, 46, -1), (0, 181, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1)):
        c.unmap(b, p, v)
    many = [new, new, 33]
    _, out, lse = attend(c, many, new)
    assert (out[2 * new:] == 0).all() and torch.isinf(lse[2 * new:]).all()        # all of it gone
    attend(c, many, new, 300, 5)


@WIDE
def test_peaked_scores_far_apart_with_many_rows(hq, hkv, new):
    attend(Cache4([3000], hq, hkv, seed=5, spread=2.0, mean=-15.0), [new], new, spread=20.0)
    attend(Cache4([700], hq, hkv, seed=6, spread=2.0, mean=-15.0), [new], new, 333, 2, spread=20.0)


@WIDE
@pytest.mark.parametrize("n,window", [(1500, NONE), (1500, 700), (400, NONE)])
def test_large_queries_with_many_rows(hq, hkv, new, n, window):
    """Scores of 1e30 and more: finite, one token's value."""
    import paper_2502_02770_amd as T
    c, G = Cache4([n], hq, hkv, seed=8), hq // hkv
    q = (queries(new, hq, 8).float() * 1e28).to(torch.bfloat16)
    out, lse = sent(q, hq)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, new, window, 0, out, lse, workspace(c.kv, new))
    for h in range(hq):
        k = c.rows(0, 0, h // G)
        x = torch.where(c.see(0, new, window, 0), (q[:, h].double() @ k.T) / math.sqrt(128), torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
        sc, ze = c.bands(0, h // G)
        # a score is off by 48 half-steps of its terms' magnitudes: rows whose two largest lie nearer have either's value or one between
        off = 48 * 2.0**-24 * (q[:, h].double().abs() @ (271 * sc + ze).T).amax(1) / math.sqrt(128)
        top = x.topk(2, 1)
        clear = top.values[:, 0] - top.values[:, 1] > 2 * off
        assert clear.float().mean() > 0.9
        want = c.rows(1, 0, h // G)[top.indices[:, 0]]
        err = (out[:, h].double() - want).abs() - ((2.0**-8 + 2 * 2.0**-11) * want.abs() + 2.0**-24)
        assert torch.isfinite(out[:, h]).all() and (err[clear] <= 0).all()
        assert ((lse[:, h].double() - top.values[:, 0]).abs() <= off + 2.0**-20 * top.values[:, 0].abs()).all()


@WIDE
def test_a_query_that_is_not_finite_spoils_only_its_row_of_many(hq, hkv, new):
    """The rows beside it stay within their bounds; not bit for bit, as the rows of a wave move their maxima together: a row's is then nearer to
    its scores' (11 below, where it may be up to 15 below), its weights smaller by that power of 2 and rounded at other places, by no more of
    themselves: what `check` allows is counted for 11, and for weights that are less than 2^-25 of the largest."""
    import paper_2502_02770_amd as T
    for n, window in ((2600, NONE), (400, 150)):
        c = Cache4([n, 90], hq, hkv, seed=9)
        many = [new, 40]
        good = queries(2 * new, hq, 9)
        q = good.clone()
        q[1, 5, 7], q[new - 1, 0, 0], q[new + 39, hq - 1, 127] = math.nan, math.inf, -math.inf
        outs = []
        for x in (good, q):
            outs.append(sent(x, hq))
            T.twilight_kv4_attention(c.kv, c.vc, c.vm, x, i32(many), i32([0, new]), new, window, 0, *outs[-1], workspace(c.kv, new))
        (want, wl), (out, lse) = outs
        bad = torch.zeros(2 * new, hq, dtype=torch.bool, device="cuda")
        bad[1, 5] = bad[new - 1, 0] = bad[new + 39, hq - 1] = True
        assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
        out[bad], lse[bad] = want[bad], wl[bad]
        for o, l in outs:
            check(c, many, [0, new], good, o, l, window, 0, (torch.full_like(o, 7.0), torch.full_like(l, 7.0)))
