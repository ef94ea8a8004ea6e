"""The cache in 4 bits: rows written and read back, and attention over it, against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.kv4_util import Cache4, unpack, values
from tests.test_gpu_new_tokens import i32, layout, queries, sent

pytestmark = pytest.mark.gpu
NONE = 2**31 - 1


def workspace(kv, max_new):
    import paper_2502_02770_amd as T
    ws = torch.empty(T.twilight_workspace_bytes(T.TW_WS_KV4, kv, max_new), dtype=torch.uint8, device="cuda")
    return ws.fill_(255)                                           # needs no clearing: NaN patterns everywhere


def reference(c, b, q, see):
    """q [N, Hq, 128] bf16, see [N, len] -> (out, lse, bound of out, bound of lse) in float64.

    Bounds.  A group's product is 32 terms q (128 + c) and one of -128 q summed, in fp32: 34 half-steps of a sum of magnitudes of at
    most 271 |q| per dim, times the scale; Q_g is summed in 8 steps, z (or z - 128 s, a rounding of 2^-24 of 128 s) times it added, 12
    more half-steps of the same magnitudes: 48 in all, and the last fma and exp2 a few of the exponent's size; so a weight is off by a
    relative e.  Weights and V are rounded to fp16 (2^-11 each; below the normal numbers by 2^-25, which for weights is 2^-36 of the
    largest, as that is at least 2^11), sums run over n terms in fp32, the output is rounded to bf16 (2^-8 of itself)."""
    N, G, n = q.shape[0], c.hq // c.hkv, c.lens[b]
    out = torch.zeros(N, c.hq, 128, dtype=torch.float64, device="cuda")
    lse = torch.full((N, c.hq), -math.inf, dtype=torch.float64, device="cuda")
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    if n == 0 or N == 0:
        return out, lse, bo, bl
    f = 1 / math.sqrt(128)
    for h in range(c.hq):
        if h % G == 0:
            kk, vv, (sc, ze) = c.rows(0, b, h // G), c.rows(1, b, h // G), c.bands(b, h // G)
        qq = q[:, h].double()
        x = torch.where(see, (qq @ kk.T) * f, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
        mag = torch.where(see, (qq.abs() @ (271 * sc + ze).T) * f, torch.zeros((), dtype=torch.float64, device="cuda")).amax(1)
        l = torch.logsumexp(x, 1)
        fin = torch.where(l == -math.inf, torch.zeros_like(l), l)
        w = torch.where(see, torch.exp(x - fin[:, None]), torch.zeros_like(x))
        top = x.abs().where(see, torch.zeros_like(x)).amax(1)
        e = 48 * 2.0**-24 * mag + 8 * 2.0**-24 * (top + 1)
        out[:, h], lse[:, h] = w @ vv, l
        bo[:, h] = (2.0**-8 * out[:, h].abs() + (2 * 2.0**-11 + 2 * e + (n + 300) * 2.0**-24)[:, None] * (w @ vv.abs())
                    + n * 2.0**-36 * w.amax(1)[:, None] * vv.abs().amax(0) + 2.0**-24)
        bl[:, h] = e + (n + 300) * 2.0**-24 + 2.0**-21 * (1 + fin.abs())
    return out, lse, bo, bl


def check(c, many, off, q, out, lse, window, sinks, before=None):
    rows = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, m in enumerate(many):
        r = slice(off[b], off[b] + m)
        rows[r] = True
        o, l, bo, bl = reference(c, b, q[r], c.see(b, m, window, sinks))
        g, gl = out[r].double(), lse[r].double()
        assert torch.isfinite(g).all(), (b, "rows")
        assert m == 0 or ((g - o).abs() - bo).max().item() <= 0, (b, ((g - o).abs() - bo).max().item())
        assert torch.equal(torch.isinf(gl), torch.isinf(l)), b
        fin = torch.isfinite(l)
        assert ((gl - l).abs()[fin] <= bl[fin]).all(), (b, (gl - l).abs()[fin].max().item())
    if before is not None:                                         # rows of no token are left
        assert torch.equal(out[~rows], before[0][~rows]) and torch.equal(lse[~rows], before[1][~rows])


def attend(c, many, max_new, window=NONE, sinks=0, seed=0, gap=0, order=None, counted=True, spread=2.0):
    import paper_2502_02770_amd as T
    off, rows = layout(many, gap, order)
    q = queries(rows, c.hq, seed, spread)
    out, lse = sent(q, c.hq)
    before = out.clone(), lse.clone()
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, i32(many) if counted else None, i32(off) if counted else None, max_new, window, sinks, out, lse,
                             workspace(c.kv, max_new))
    check(c, many, off, q, out, lse, window, sinks, before)
    return q, out, lse


HEADS = [(8, 8), (8, 4), (32, 8), (16, 2), (8, 1)]


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n", [1, 15, 16, 17, 64, 65, 255, 256, 257, 1000, 4099])
def test_one_token(hq, hkv, n):
    attend(Cache4([n], hq, hkv, seed=n), [1], 1, seed=n, counted=False)


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("new", [2, 3, 5, 8, 13, 16, 33, 100])
def test_drafts_and_chunks(hq, hkv, new):
    lens = [new, new + 1, 300, 1031]
    many = [new, 1, min(new, 300), max(1, new - 1)]
    attend(Cache4(lens, hq, hkv, seed=new), many, new, seed=new, gap=2, order=[2, 0, 3, 1])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (17, 16), (63, 17), (64, 0), (129, 70), (500, 3), (4000, 64), (NONE, 5)])
@pytest.mark.parametrize("new,hq,hkv", [(1, 16, 4), (7, 16, 4), (40, 8, 8)])
def test_windows(window, sinks, new, hq, hkv):
    lens = [40, 513, 1700, 65]
    attend(Cache4(lens, hq, hkv, seed=window % 1000 + sinks), [min(new, n) for n in lens], new, window, sinks, seed=sinks)


def test_empty_sequences_and_none_new():
    attend(Cache4([0, 5, 700, 0], 16, 4, max_pages=50), [1, 0, 1, 0], 1)
    attend(Cache4([0, 3, 700], 16, 4, max_pages=50), [0, 0, 0], 4)


def test_more_new_tokens_than_the_sequence_has():
    """Those before position 0 see nothing: rows of zeros."""
    c = Cache4([3, 40], 16, 4)
    q, out, lse = attend(c, [9, 9], 9)
    assert (out[:6] == 0).all() and torch.isinf(lse[:6]).all()


def test_pages_that_are_not_there():
    c = Cache4([700, 64, 33], 16, 4)
    for b, p, v in ((0, 0, -1), (0, 7, 1 << 30), (0, 43, -5), (1, 0, -1), (1, 1, -1), (1, 2, -1), (1, 3, -1), (2, 2, -1)):
        c.unmap(b, p, v)
    _, out, lse = attend(c, [1, 1, 1], 1)
    assert (out[1] == 0).all() and torch.isinf(lse[1]).all()       # all of it gone
    attend(c, [20, 20, 20], 20, 300, 5)


def test_ragged_batch_of_many():
    rng = np.random.default_rng(3)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(3000), 70))]
    many = [int(rng.integers(0, min(4, n) + 1)) for n in lens]
    attend(Cache4(lens, 8, 2, seed=3), many, 4, seed=3)


def test_long_context():
    attend(Cache4([70001], 8, 2, seed=1), [1], 1)
    attend(Cache4([40000, 9], 8, 1, seed=2), [12, 2], 12, 30000, 9)


def test_a_prompt_and_single_tokens():
    attend(Cache4([900, 2000, 17, 5000], 16, 2, seed=4), [900, 1, 1, 1], 900)


def test_peaked_scores_far_apart():
    """Scores of some hundreds: one token takes all, and the running maximum moves by far more than fp16 reaches."""
    attend(Cache4([3000], 16, 4, seed=5, spread=2.0, mean=-15.0), [6], 6, spread=20.0)


def test_even_weights_behind_a_large_one():
    """65535 tokens of weight 2^-16 of the largest, together as much as it: none may be lost to fp16."""
    n = 65536
    c = Cache4([n], 8, 1, seed=6)
    c.kc.zero_()
    c.km[..., 0], c.km[..., 1] = 0.0, 0.0
    h = c.table[0, 100].item()
    c.km[h, :, 3, 0, 1] = 1.0
    q = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    q[:, :, :32] = 16 * math.log(2) * math.sqrt(128) / 32
    import paper_2502_02770_amd as T
    out, lse = sent(q, 8)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 1, NONE, 0, out, lse, workspace(c.kv, 1))
    check(c, [1], [0], q, out, lse, NONE, 0)


@pytest.mark.parametrize("v", [1e-6, 1e-4, 1.0, 2.9e4])
def test_sizes_of_values(v):
    """V from the smallest fp16 numbers to the largest that a row may have."""
    c = Cache4([777], 16, 4, seed=7)
    scale = v / 16
    c.vm[..., 0] = torch.where(torch.isnan(c.vm[..., 0]), c.vm[..., 0], torch.full_like(c.vm[..., 0], scale))
    c.vm[..., 1] = torch.where(torch.isnan(c.vm[..., 1]), c.vm[..., 1], torch.full_like(c.vm[..., 1], -v / 2))
    attend(c, [3], 3)


def test_large_queries():
    """Scores of 1e30 and more: finite, one token's value."""
    import paper_2502_02770_amd as T
    c = Cache4([500], 8, 2, seed=8)
    q = (queries(2, 8, 8).float() * 1e28).to(torch.bfloat16)
    out, lse = sent(q, 8)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 2, NONE, 0, out, lse, workspace(c.kv, 2))
    for h in range(8):
        x = (q[:, h].double() @ c.rows(0, 0, h // 4).T) / math.sqrt(128)
        x = torch.where(c.see(0, 2, NONE, 0), x, torch.full_like(x, -math.inf))
        best = x.argmax(1)
        want = c.rows(1, 0, h // 4)[best]
        assert ((out[:, h].double() - want).abs() <= (2.0**-8 + 2 * 2.0**-11) * want.abs() + 2.0**-24).all()
        assert ((lse[:, h].double() / x.amax(1) - 1).abs() <= 1e-5).all()


def test_a_query_that_is_not_finite_spoils_only_its_row():
    import paper_2502_02770_amd as T
    c = Cache4([600, 90], 16, 4, seed=9)
    q = queries(6, 16, 9)
    ws = workspace(c.kv, 3)
    out, lse = sent(q, 16)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 3, NONE, 0, out, lse, ws)
    want, wl = out.clone(), lse.clone()
    q[1, 5, 7], q[4, 0, 0] = math.nan, math.inf
    out, lse = sent(q, 16)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 3, NONE, 0, out, lse, ws)
    bad = torch.zeros(6, 16, dtype=torch.bool, device="cuda")
    bad[1, 5] = bad[4, 0] = True
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], wl[~bad])


def test_lse_is_optional_and_calls_repeat_bit_for_bit():
    import paper_2502_02770_amd as T
    c = Cache4([5000, 333], 32, 8, seed=10)
    q, out, lse = attend(c, [2, 2], 2, seed=10)
    ws = workspace(c.kv, 2)
    for _ in range(3):
        again = torch.zeros_like(out)
        T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, i32([2, 2]), i32([0, 2]), 2, NONE, 0, again, None, ws)
        assert torch.equal(again, out)


def test_offsets_beyond_32_bits():
    """Codes further than 2^32 bytes into the pools."""
    shift = (1 << 32) // (8 * 1024) + 5
    c = Cache4([300, 40], 8, 8, seed=11, shift=shift)
    attend(c, [2, 1], 2)


def test_streams_and_a_graph():
    """Calls on two streams at once, each with its workspace; captured and replayed over a cache that grows."""
    import paper_2502_02770_amd as T
    c = Cache4([3000, 800], 16, 4, seed=12)
    q = queries(2, 16, 12)
    want, wl = sent(q, 16)
    T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 1, NONE, 0, want, wl, workspace(c.kv, 1))
    torch.cuda.synchronize()
    streams, outs, ws = [torch.cuda.Stream() for _ in range(2)], [sent(q, 16) for _ in range(2)], [workspace(c.kv, 1) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (o, l), w in zip(streams, outs, ws):
            with torch.cuda.stream(s):
                T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 1, NONE, 0, o, l, w)
    torch.cuda.synchronize()
    for o, l in outs:
        assert torch.equal(o, want) and torch.equal(l, wl)
    g, (o, l) = torch.cuda.CUDAGraph(), outs[0]
    with torch.cuda.graph(g):
        T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 1, NONE, 0, o, l, ws[0])
    for n in ([3000, 800], [2999, 17], [1, 800], [3000, 0]):
        c.seq.copy_(i32(n))
        g.replay()
        e, el = sent(q, 16)
        T.twilight_kv4_attention(c.kv, c.vc, c.vm, q, None, None, 1, NONE, 0, e, el, ws[1])
        assert torch.equal(o, e) and torch.equal(l, el)


# --------------------------------------------------------------------------------------------------- rows written, read back
def _store(lens, many, hkv, seed, bounds=True, max_pages=None):
    """A cache that holds lens[b] tokens, and many[b] new rows for each."""
    full = [n + m for n, m in zip(lens, many)]
    c = Cache4(full, hkv, hkv, seed=seed, max_pages=max_pages)
    c.bounds = (torch.randn(c.kc.shape[0], hkv, 2, 128, device="cuda") * 0.1).to(torch.bfloat16) if bounds else None
    rows = max(1, sum(many))
    k = (torch.randn(rows, hkv, 128, device="cuda") * 2 + 1).to(torch.bfloat16)
    v = (torch.randn(rows, hkv, 128, device="cuda") * 0.1 - 3).to(torch.bfloat16)
    return c, k, v


@pytest.mark.parametrize("hkv", [1, 4, 8])
@pytest.mark.parametrize("lens,many", [([0], [1]), ([5], [1]), ([16], [1]), ([15, 0, 31], [2, 17, 1]), ([7, 100, 0], [300, 0, 33]), ([0, 40], [1000, 7])])
def test_append_is_kquant_append_for_k_and_for_v(lens, many, hkv):
    """Codes, (scale, zero) and bounds bit for bit those that twilight_kquant_append leaves, of V as if V were K."""
    import paper_2502_02770_amd as T
    c, k, v = _store(lens, many, hkv, seed=sum(lens))
    off = i32(np.cumsum([0] + many[:-1]).tolist())
    want = []
    for x in (k, v):
        codes, meta, bounds = c.kc.clone(), c.km.clone(), c.bounds.clone()
        kv = T.make_kv(len(lens), hkv, hkv, c.max_pages, c.kc.shape[0], c.table, c.seq, None, None, codes, meta, bounds)
        T.twilight_kquant_append(kv, x, None, i32(lens), i32(many), off, max(many))
        want.append((codes, meta, bounds))
    got = [c.kc.clone(), c.km.clone(), c.kc.clone(), c.km.clone(), c.bounds.clone()]
    kv = T.make_kv(len(lens), hkv, hkv, c.max_pages, c.kc.shape[0], c.table, c.seq, None, None, got[0], got[1], got[4])
    T.twilight_kv4_append(kv, got[2], got[3], k, v, i32(lens), i32(many), off, max(many))
    bits = lambda t: t.view(torch.int16) if t.dtype != torch.uint8 else t
    for a, b in zip(got, (want[0][0], want[0][1], want[1][0], want[1][1], want[0][2])):
        assert torch.equal(bits(a), bits(b))


def test_append_of_zeros_of_both_signs_and_of_the_smallest_numbers():
    """The least and the largest are found on the numbers' bits: what compares equal or is below the normal range has to come out alike."""
    import paper_2502_02770_amd as T
    c, k, v = _store([3], [40], 2, seed=8)
    g = torch.Generator("cuda").manual_seed(8)
    small = torch.tensor([0, -0x8000, 1, -0x7FFF, 0x7F, -0x7F81, 0x80, -0x7F80], dtype=torch.int16, device="cuda").view(torch.bfloat16)
    for x, many in ((k, 2), (v, 8)):
        x.copy_(small[torch.randint(0, many, x.shape, device="cuda", generator=g)])
    got = [c.kc.clone(), c.km.clone(), c.kc.clone(), c.km.clone(), c.bounds.clone()]
    want = [t.clone() for t in got]
    make = lambda codes, meta, bounds: T.make_kv(1, 2, 2, c.max_pages, c.kc.shape[0], c.table, c.seq, None, None, codes, meta, bounds)
    T.twilight_kquant_append(make(want[0], want[1], want[4]), k, None, i32([3]), i32([40]), i32([0]), 40)
    T.twilight_kquant_append(make(want[2], want[3], torch.zeros_like(want[4])), v, None, i32([3]), i32([40]), i32([0]), 40)
    T.twilight_kv4_append(make(got[0], got[1], got[4]), got[2], got[3], k, v, i32([3]), i32([40]), i32([0]), 40)
    bits = lambda t: t.view(torch.int16) if t.dtype != torch.uint8 else t
    for a, b in zip(got, want):
        assert torch.equal(bits(a), bits(b))


def test_append_to_pages_that_are_not_there_and_without_bounds():
    import paper_2502_02770_amd as T
    c, k, v = _store([0], [100], 2, seed=1, bounds=False)
    c.unmap(0, 2)
    c.unmap(0, 4, 1 << 30)
    before = [x.clone() for x in (c.kc, c.km, c.vc, c.vm)]
    T.twilight_kv4_append(c.kv, c.vc, c.vm, k, v, i32([0]), i32([100]), i32([0]), 64)          # counts are cut to max_new
    held = c.table[0, [0, 1, 3]].long()
    other = torch.ones(c.kc.shape[0], dtype=torch.bool, device="cuda")
    other[held] = False
    for a, b in zip((c.kc, c.km, c.vc, c.vm), before):
        assert torch.equal(a[other].view(torch.uint8), b[other].view(torch.uint8)) and not torch.equal(a[held].view(torch.uint8), b[held].view(torch.uint8))
    T.twilight_kv4_append(c.kv, c.vc, c.vm, k, v, i32([0]), i32([100]), i32([0]), 0)
    T.twilight_kv4_append(c.kv, c.vc, c.vm, k, v, i32([-3]), i32([100]), i32([0]), 100)        # no position: nothing


@pytest.mark.parametrize("hkv", [1, 8])
def test_rows_read_back(hkv):
    """Every row the bf16 number next to code * scale + zero; rows behind a sequence's end left, rows of missing pages zero."""
    import paper_2502_02770_amd as T
    lens = [40, 333, 16, 0]
    c = Cache4(lens, hkv, hkv, seed=2, max_pages=30)
    c.unmap(1, 3)
    start, many, off = [3, 0, 15, 0], [50, 333, 1, 9], [1, 60, 400, 410]
    k = torch.full((420, hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    T.twilight_kv4_read(c.kv, c.vc, c.vm, i32(start), i32(many), i32(off), 333, k, v)
    for which, got in ((0, k), (1, v)):
        want = torch.full((420, hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        for b, n in enumerate(lens):
            m = max(0, min(many[b], n - start[b]))
            for h in range(hkv):
                if n:
                    want[off[b]:off[b] + m, h] = c.rows(which, b, h)[start[b]:start[b] + m].float().to(torch.bfloat16)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_written_rows_are_within_half_a_step():
    """Append, read: off by half a step of the codes, the rounding of (scale, zero), and of the bf16 row."""
    import paper_2502_02770_amd as T
    c, k, v = _store([0, 9], [200, 77], 4, seed=3)
    T.twilight_kv4_append(c.kv, c.vc, c.vm, k, v, i32([0, 9]), i32([200, 77]), i32([0, 200]), 200)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    T.twilight_kv4_read(c.kv, c.vc, c.vm, i32([0, 9]), i32([200, 77]), i32([0, 200]), 200, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        g = x.double().reshape(*x.shape[:2], 4, 32)
        step = (g.amax(-1) - g.amin(-1)) / 15
        bound = 0.5 * step * (1 + 2.0**-10) + 16 * step * 2.0**-11 + g.abs().amax(-1) * (2.0**-11 + 2.0**-8)
        assert ((y.double().reshape(g.shape) - g).abs() <= bound[..., None]).all()


# ------------------------------------------------------------------------------------------------------------ a run of them
def test_a_sequence_in_four_bits_from_prompt_to_tokens():
    """PagedKV4: prompt appended and attended, then tokens one at a time, a fork's pages copied, a row read back."""
    import paper_2502_02770_amd as T
    B, hq, hkv, pages = 2, 8, 2, 12
    table = torch.full((B, pages), -1, dtype=torch.int32)
    cache = T.PagedKV4(hq, hkv, table, torch.zeros(B, dtype=torch.int32), 40)
    pool = T.PagePool(cache)
    lens, max_new = [0, 0], 70
    g = torch.Generator("cuda").manual_seed(0)
    rand = lambda n, h: torch.randn(n, h, 128, device="cuda", generator=g).to(torch.bfloat16)
    for many in ([70, 33], [1, 1], [1, 0], [5, 1], [1, 1]):
        step, off = NewTokensOf(cache, max(many)), [b * max(many) for b in range(B)]
        pool.reserve(i32(many), max(many))
        k, v, q = (rand(B * max(many), h) for h in (hkv, hkv, hq))
        cache.append(k, v, cache.seq_lens.clone(), i32(many), i32(off), max(many))
        lens = [n + m for n, m in zip(lens, many)]
        cache.seq_lens.copy_(i32(lens))
        out = step.window(q, NONE, 0, i32(many))
        ref = _view(cache, lens)
        check(ref, many, off, q, out, step.lse, NONE, 0)
    new_table, new_lens, src, dst = pool.fork(i32([0, 0, 1]))
    cache.copy_pages(src, dst)
    child = cache.over(new_table, new_lens)
    step = NewTokensOf(child, 1)
    q = rand(3, hq)
    out = step.window(q, 20, 4)
    check(_view(child, [lens[0], lens[0], lens[1]]), [1, 1, 1], [0, 1, 2], q, out, step.lse, 20, 4)
    with pytest.raises(AssertionError):
        step.tree(q, torch.zeros(3, 1, dtype=torch.int32, device="cuda"))
    ko, vo = torch.empty(9, hkv, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(9, hkv, 128, dtype=torch.bfloat16, device="cuda")
    child.read(i32([0, 4, 30]), i32([3, 3, 3]), i32([0, 3, 6]), 3, ko, vo)
    ref = _view(child, [lens[0], lens[0], lens[1]])
    for b, at in enumerate((0, 4, 30)):
        for h in range(hkv):
            assert torch.equal(ko[3 * b:3 * b + 3, h], ref.rows(0, b, h)[at:at + 3].float().to(torch.bfloat16))
            assert torch.equal(vo[3 * b:3 * b + 3, h], ref.rows(1, b, h)[at:at + 3].float().to(torch.bfloat16))


def NewTokensOf(cache, n):
    import paper_2502_02770_amd as T
    return T.NewTokens(cache, n)


def _view(cache, lens):
    """What tests/kv4_util.py reads of a cache, of a PagedKV4."""
    c = object.__new__(Cache4)
    c.lens, c.hq, c.hkv, c.table, c.unmapped = lens, cache.Hq, cache.Hkv, cache.page_table, {}
    c.pools = [(cache.kq_pool, cache.kq_meta), (cache.vq_pool, cache.vq_meta)]
    (c.kc, c.km), (c.vc, c.vm) = c.pools
    return c


def test_codes_of_the_pools_are_read_as_documented():
    """The helper's reading of a packed row against the one of the append tests of bf16 caches."""
    from tests.gpu_util import unpack_codes
    x = torch.randint(0, 256, (5, 64), dtype=torch.uint8)
    assert np.array_equal(unpack(x).numpy().astype(np.uint8), unpack_codes(x.numpy(), 4))
    assert values(x, torch.ones(5, 4, 2).half()).shape == (5, 128)
