"""Attention of several new tokens per sequence (drafted trees, sliding windows with sinks) against its definition in 64
bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
NONE = 2**31 - 1


class Cache:
    """A paged cache with shuffled pages; rows that are no token, and pages that no table names, hold NaN."""

    def __init__(self, lens, hq, hkv, seed=0, max_pages=None, spare=3, shift=0):
        import paper_2502_02770_amd as T
        g = torch.Generator("cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        held = [-(-n // 16) for n in lens]
        self.lens, self.hq, self.hkv = lens, hq, hkv
        P = sum(held) + spare + shift
        ids = rng.permutation(sum(held) + spare) + shift
        self.max_pages = max_pages or max(1, max(held))
        table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for b, h in enumerate(held):
            table[b, :h] = ids[at:at + h]
            at += h
        self.table = torch.from_numpy(table).cuda()
        self.k = torch.empty(P, hkv, 16, 128, dtype=torch.bfloat16, device="cuda")
        self.v = torch.empty_like(self.k)
        self.k[shift:], self.v[shift:] = math.nan, math.nan
        self.logical = []
        for b, n in enumerate(lens):
            k = torch.randn(held[b] * 16, hkv, 128, device="cuda", generator=g, dtype=torch.bfloat16)
            v = torch.randn(held[b] * 16, hkv, 128, device="cuda", generator=g, dtype=torch.bfloat16) + 0.5
            k[n:], v[n:] = math.nan, math.nan
            p = self.table[b, :held[b]].long()
            self.k[p] = k.view(-1, 16, hkv, 128).transpose(1, 2)
            self.v[p] = v.view(-1, 16, hkv, 128).transpose(1, 2)
            self.logical.append((k[:n], v[:n]))
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.kv = T.make_kv(len(lens), hq, hkv, self.max_pages, P, self.table, self.seq, self.k, self.v)

    def unmap(self, b, page, value=-1):
        """Takes a page away: nobody sees its tokens."""
        self.table[b, page] = value
        return set(range(page * 16, page * 16 + 16))


def reference(cache, b, q, see):
    """q [N, Hq, 128] bf16, see [N, len] truth values -> (out, lse, bound of out, bound of lse) in float64.

    Bounds: a score is 128 products summed in fp32 (130 half-steps of the sum of their magnitudes), then one fma and exp2
    (a few steps of the exponent's size); so a weight is off by a relative e.  Weights are rounded to bf16 for the product
    with V (2^-8 of each), sums run over n terms in fp32, the output is rounded to bf16 (2^-8 of itself)."""
    N, G = q.shape[0], cache.hq // cache.hkv
    n = cache.lens[b]
    out = torch.zeros(N, cache.hq, 128, dtype=torch.float64, device="cuda")
    lse = torch.full((N, cache.hq), -math.inf, dtype=torch.float64, device="cuda")
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    if n == 0 or N == 0:
        return out, lse, bo, bl
    k, v = cache.logical[b]
    s = 1 / math.sqrt(128)
    for h in range(cache.hq):
        kk, vv, qq = k[:, h // G].double(), v[:, h // G].double(), q[:, h].double()
        x = (qq @ kk.T) * s
        mag = (qq.abs() @ kk.abs().T) * s
        x = torch.where(see, x, torch.full_like(x, -math.inf))
        mag = torch.where(see, mag, torch.zeros_like(mag)).amax(1)
        l = torch.logsumexp(x, 1)
        w = torch.where(see, torch.exp(x - torch.where(l == -math.inf, torch.zeros_like(l), l)[:, None]), torch.zeros_like(x))
        e = 130 * 2.0**-24 * mag + 8 * 2.0**-24 * (mag + 1)
        out[:, h], lse[:, h] = w @ vv, l
        bo[:, h] = 2.0**-8 * out[:, h].abs() + (2.0**-8 + 2 * e + (n + 300) * 2.0**-24)[:, None] * (w @ vv.abs())
        bl[:, h] = e + (n + 300) * 2.0**-24 + 2.0**-21 * (1 + torch.where(l == -math.inf, torch.zeros_like(l), l).abs())
    return out, lse, bo, bl


def check(cache, many, offsets, q, out, lse, see_of, before=None):
    rows = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, m in enumerate(many):
        r = slice(offsets[b], offsets[b] + m)
        rows[r] = True
        o, l, bo, bl = reference(cache, b, q[r], see_of(b, m))
        g, gl = out[r].double(), lse[r].double()
        assert torch.isfinite(g).all(), (b, "rows")
        worst = ((g - o).abs() - bo).max().item() if m else 0
        assert worst <= 0, (b, worst)
        assert torch.equal(torch.isinf(gl), torch.isinf(l)), b
        fin = torch.isfinite(l)
        assert ((gl - l).abs()[fin] <= bl[fin]).all(), (b, (gl - l).abs()[fin].max().item())
    if before is not None:                                         # rows of no token are left
        assert torch.equal(out[~rows], before[0][~rows]) and torch.equal(lse[~rows], before[1][~rows])


def sent(q, hq):
    return torch.full_like(q, 7.0), torch.full((q.shape[0], hq), 7.0, dtype=torch.float32, device="cuda")


def layout(many, gap=0, order=None):
    """Row of each sequence's first new token: in the given order, `gap` rows between; total rows."""
    off, at = [0] * len(many), gap
    for b in (order if order is not None else range(len(many))):
        off[b] = at
        at += many[b] + gap
    return off, max(1, at)


def queries(rows, hq, seed, spread=2.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(rows, hq, 128, device="cuda", generator=g) * spread).to(torch.bfloat16)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def workspace(kv, max_new):
    import paper_2502_02770_amd as T
    ws = torch.empty(T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, kv, max_new), dtype=torch.uint8, device="cuda")
    return ws.fill_(255)                                           # needs no clearing: NaN patterns everywhere


def run_tree(cache, many, max_new, seed=0, gap=0, order=None, density=None, words=None, offsets=True, holes=None, spread=2.0):
    import paper_2502_02770_amd as T
    rng = np.random.default_rng(seed)
    off, rows = layout(many, gap, order)
    words = words or -(-max_new // 32)
    bits = np.zeros((rows, words * 32), dtype=np.uint8)
    if density is None:                                            # random trees
        for b, m in enumerate(many):
            for j in range(m):
                up = int(rng.integers(-1, j)) if j else -1
                if up >= 0:
                    bits[off[b] + j, :m] = bits[off[b] + up, :m]
                bits[off[b] + j, j] = 1
    else:                                                          # any mask at all, bits beyond the draft too
        bits[:] = rng.random(bits.shape) < density
    mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).cuda()
    q = queries(rows, cache.hq, seed + 1, spread)
    out, lse = sent(q, cache.hq)
    before = out.clone(), lse.clone()
    T.twilight_tree_attention(cache.kv, q, i32(many) if offsets else None, i32(off) if offsets else None, max_new, mask, words, out, lse,
                              workspace(cache.kv, max_new))
    holes = holes or {}

    def see(b, m):
        n = cache.lens[b]
        s = np.zeros((m, max(n, 1)), dtype=bool)[:, :n]
        ctx = n - m
        s[:, :max(ctx, 0)] = True
        for j in range(max(0, -ctx), m):
            s[:, ctx + j] = bits[off[b]:off[b] + m, j]
        s[:, sorted(t for t in holes.get(b, ()) if t < n)] = False
        return torch.from_numpy(s).cuda()

    check(cache, many, off, q, out, lse, see, before)
    return out, lse


def run_window(cache, many, max_new, window, sinks, seed=0, gap=0, order=None, offsets=True, holes=None, spread=2.0):
    import paper_2502_02770_amd as T
    off, rows = layout(many, gap, order)
    q = queries(rows, cache.hq, seed + 1, spread)
    out, lse = sent(q, cache.hq)
    before = out.clone(), lse.clone()
    T.twilight_window_attention(cache.kv, q, i32(many) if offsets else None, i32(off) if offsets else None, max_new, window, sinks, out, lse,
                                workspace(cache.kv, max_new))
    holes = holes or {}

    def see(b, m):
        n = cache.lens[b]
        p = torch.arange(n - m, n, device="cuda")[:, None]
        t = torch.arange(n, device="cuda")[None]
        s = (t <= p) & ((p - t < window) | (t < sinks))
        s[:, sorted(x for x in holes.get(b, ()) if x < n)] = False
        return s

    check(cache, many, off, q, out, lse, see, before)
    return out, lse


HEADS = [(8, 8), (8, 4), (8, 2), (16, 2)]                          # groups of 1, 2, 4, 8 query heads


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("max_new", [1, 5, 17, 61, 100])
def test_trees_of_ragged_batches(hq, hkv, max_new):
    rng = np.random.default_rng(max_new)
    lens = [1, 15, 16, 17, 63, 64, 65, 500, 1031]
    many = [min(n, int(rng.integers(0, max_new + 1))) for n in lens]
    many[3], many[-1] = min(17, max_new), max_new
    run_tree(Cache(lens, hq, hkv, seed=max_new), many, max_new, seed=max_new, gap=2, order=rng.permutation(len(lens)))


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("max_new", [1, 12, 40, 130])
def test_short_sequences_in_wide_tables(hq, hkv, max_new):
    """Rows of the page table could hold long sequences: the lists are planned on the device, and may be cut or not."""
    lens = [1, 64, 200, 1500, 0, 130]
    c = Cache(lens, hq, hkv, seed=max_new, max_pages=1000)
    many = [min(n, max_new) for n in lens]
    run_tree(c, many, max_new, seed=1)
    run_window(c, many, max_new, 500, 3, seed=2)
    run_window(c, many, max_new, NONE, 0, seed=3)


def test_values_offloaded_to_the_host():
    """K and V in pinned host memory, read over the link."""
    import paper_2502_02770_amd as T
    c = Cache([90, 300], 8, 2, seed=20)
    far = T.PagedKV(8, 2, c.table, c.seq, c.k.shape[0], "cuda", offload_kv=True)
    far.k_pool.copy_(c.k)
    far.v_pool.copy_(c.v)
    c.kv = far.kv
    run_tree(c, [7, 40], 40)
    run_window(c, [7, 40], 40, 100, 5)


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("density", [0.0, 0.1, 0.7])
def test_trees_with_any_mask(hq, hkv, density):
    """Rows that see nothing (no context), no ancestor, not themselves; bits of tokens beyond the draft."""
    run_tree(Cache([40, 3, 130, 7], hq, hkv, seed=3), [40, 3, 37, 0], 40, seed=5, density=density, words=3)


def test_a_draft_longer_than_its_sequence():
    run_tree(Cache([9, 33], 8, 2, seed=1), [20, 33], 33, density=0.5)


@pytest.mark.parametrize("max_new", [1, 64, 300, 1024])
def test_one_tree_over_a_long_cache(max_new):
    run_tree(Cache([20011], 8, 2, seed=2), [max_new], max_new, seed=max_new)


def test_empty_sequences_and_no_drafts():
    run_tree(Cache([0, 5, 0, 100], 8, 2, seed=4, max_pages=9), [0, 0, 4, 1], 4, density=1.0)
    run_window(Cache([0, 5, 0, 100], 8, 2, seed=4, max_pages=9), [0, 0, 0, 1], 4, 10, 2)


@pytest.mark.parametrize("value", [-1, 10**9, -2**31])
def test_unmapped_pages_are_seen_by_nobody(value):
    c = Cache([300, 200, 16], 8, 2, seed=6)
    holes = {0: c.unmap(0, 0, value) | c.unmap(0, 7, value) | c.unmap(0, 18, value), 2: c.unmap(2, 0, value)}
    run_tree(c, [5, 9, 2], 9, holes=holes, density=0.6)
    run_window(c, [5, 9, 2], 9, 150, 20, holes=holes)
    run_window(c, [5, 9, 2], 9, NONE, 0, holes=holes)


def test_many_sequences():
    """More than a wave of sequences in the plan, some long."""
    rng = np.random.default_rng(0)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(2000), 150))]
    lens[70], lens[149] = 6000, 3001
    c = Cache(lens, 8, 2, seed=8)
    run_tree(c, [min(n, int(rng.integers(0, 8))) for n in lens], 7, seed=9)
    run_window(c, [min(n, int(rng.integers(0, 8))) for n in lens], 7, 257, 3, seed=9)


def test_lists_of_many_tiles_in_one_piece():
    """As many lists as workgroups: a workgroup walks more tiles than it holds page ids for."""
    c = Cache([6007] * 63 + [9000], 16, 8, seed=10)
    run_tree(c, [1] * 64, 1, seed=11)


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 1), (100, 5), (1000, 70), (NONE, 0), (64, 64), (33, NONE)])
def test_windows_of_ragged_batches(hq, hkv, window, sinks):
    lens = [1, 16, 63, 65, 300, 1031, 2000]
    many = [1, 3, 63, 1, 40, 100, 77]
    run_window(Cache(lens, hq, hkv, seed=1), many, 100, window, sinks, seed=window % 97, gap=1, order=[3, 1, 0, 6, 5, 2, 4])


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 1), (4096, 4), (1000, 0), (NONE, 0)])
def test_windows_of_single_tokens(hq, hkv, window, sinks):
    lens = [1, 4, 64, 999, 1000, 1001, 9000]
    run_window(Cache(lens, hq, hkv, seed=2), [1] * 7, 1, window, sinks, offsets=False)


@pytest.mark.parametrize("hq,hkv,tokens", [(32, 8, 1031), (8, 8, 1500), (64, 8, 700)])
@pytest.mark.parametrize("window,sinks", [(200, 4), (NONE, 0), (640, 130)])
def test_windows_of_whole_prompts(hq, hkv, tokens, window, sinks):
    """Row blocks enough for the whole chip: nothing is cut."""
    lens = [tokens, tokens // 2 + 3, 1, tokens - 1]
    run_window(Cache(lens, hq, hkv, seed=3), lens, tokens, window, sinks, seed=5)


@pytest.mark.parametrize("hq,hkv,new", [(8, 8, 1), (32, 8, 5), (16, 2, 30), (8, 4, 60)])
@pytest.mark.parametrize("sinks", [1, 16, 17, 40, 63, 100])
def test_pages_of_sinks_and_pages_of_the_window_in_one_tile(hq, hkv, new, sinks):
    """The sinks' pages end inside a tile and the window begins on any page, next to them or far behind."""
    lens = [400, 129, 144, 1000, 161, 97, 15, 257, 64]
    c = Cache(lens, hq, hkv, seed=sinks)
    for window in (1, 15, 30, 64, 110):
        run_window(c, [min(n, new) for n in lens], new, window, sinks, seed=window)


def test_a_table_with_room_for_more_work_than_32_bits_count():
    """Row blocks x tiles that the arguments allow are 2^33; the sequences are short."""
    c = Cache([200, 0, 77, 1000], 64, 8, seed=3, max_pages=1 << 24)
    run_tree(c, [3, 0, 20, 9], 1024, seed=5)


@pytest.mark.parametrize("window,sinks", [(2**32 + 5, 0), (2**63 - 1, 3), (5, 2**32 + 1)])
def test_windows_and_sinks_beyond_32_bits_are_no_limit(window, sinks):
    run_window(Cache([300, 40], 8, 2, seed=6), [7, 40], 40, window, sinks)


def test_a_window_over_freed_pages():
    """Pages between the sinks and the window have been given back."""
    c = Cache([5000], 8, 2, seed=12)
    holes = {0: set()}
    for p in range(1, (5000 - 10 - 512) // 16):
        holes[0] |= c.unmap(0, p)
    run_window(c, [10], 10, 512, 16, holes=holes)


def test_a_draft_longer_than_its_sequence_under_a_window():
    import paper_2502_02770_amd as T
    c = Cache([5], 8, 2, seed=13)
    q = queries(9, 8, 1)
    out, lse = sent(q, 8)
    T.twilight_window_attention(c.kv, q, None, None, 9, 4, 0, out, lse, workspace(c.kv, 9))
    assert (out[:4] == 0).all() and (lse[:4] == -math.inf).all()   # positions below 0 see nothing
    see = torch.tril(torch.ones(5, 5, dtype=torch.bool, device="cuda")).triu(-3)
    o, l, bo, bl = reference(c, 0, q[4:], see)
    assert ((out[4:].double() - o).abs() <= bo).all() and ((lse[4:].double() - l).abs() <= bl).all()


def test_peaked_rows_and_large_scores():
    """Logits of some hundreds: one token decides a row, and the running maximum climbs from tile to tile."""
    c = Cache([700], 8, 2, seed=14)
    run_window(c, [30], 30, NONE, 0, spread=40.0)
    run_tree(c, [30], 30, spread=40.0)


def test_cache_beyond_32_bits():
    """Pools of 5 GiB, the sequence's pages at their end."""
    c = Cache([3000], 8, 8, seed=15, shift=(5 << 30) // (8 * 16 * 256))
    assert c.k.numel() * 2 > 1 << 32
    run_tree(c, [20], 20)
    run_window(c, [20], 20, 700, 5)


def test_a_long_prompt():
    """20000 tokens at once, a window of 79 tiles: some rows of every part against the definition."""
    import paper_2502_02770_amd as T
    n, W, S = 20003, 5000, 5
    c = Cache([n], 8, 2, seed=21)
    q = queries(n, 8, 1)
    out, lse = sent(q, 8)
    T.twilight_window_attention(c.kv, q, None, None, n, W, S, out, lse, workspace(c.kv, n))
    rows = torch.cat([torch.arange(a, a + 12, device="cuda") for a in (0, 58, 4990, 5060, 12345, n - 12)])
    t = torch.arange(n, device="cuda")[None]
    see = (t <= rows[:, None]) & ((rows[:, None] - t < W) | (t < S))
    o, l, bo, bl = reference(c, 0, q[rows], see)
    assert ((out[rows].double() - o).abs() <= bo).all() and ((lse[rows].double() - l).abs() <= bl).all()


def test_a_long_context():
    """Few lists of thousands of tiles."""
    c = Cache([200013], 8, 2, seed=22)
    run_tree(c, [3], 3)
    run_window(c, [40], 40, 150000, 100)


def test_a_row_that_is_not_finite_keeps_to_itself():
    import paper_2502_02770_amd as T
    c = Cache([300, 70], 8, 2, seed=23)
    q = queries(20, 8, 1)
    run = lambda q: T.twilight_window_attention(c.kv, q, None, None, 10, 100, 3, *(keep := sent(q, 8)), workspace(c.kv, 10)) or keep
    a = run(q)
    q2 = q.clone()
    q2[4, 3] = math.nan
    q2[13, 7, 5] = math.inf
    b = run(q2)
    others = torch.ones(20, 8, dtype=torch.bool, device="cuda")
    others[4, 3] = others[13, 7] = False
    assert torch.isnan(b[0][4, 3]).all() and torch.equal(a[0][others], b[0][others]) and torch.equal(a[1][others], b[1][others])
    # a drafted token whose K is not finite, hidden from the others by their masks
    p = int(c.table[1, 69 // 16])
    c.k[p, :, 69 % 16] = math.nan                                  # the last token of the second sequence
    x = run(q)
    hidden = torch.ones(20, dtype=torch.bool, device="cuda")
    hidden[19] = False                                             # only its own row sees it
    assert torch.equal(x[0][hidden], a[0][hidden]) and torch.isnan(x[0][19]).all()


def test_two_streams_at_once():
    import paper_2502_02770_amd as T
    c = Cache([5000, 40, 900], 32, 8, seed=24)
    qs = [queries(3 * 4, 32, k) for k in (1, 2)]
    ws = [workspace(c.kv, 4) for _ in qs]
    alone, both = [sent(q, 32) for q in qs], [sent(q, 32) for q in qs]
    for q, o, w in zip(qs, alone, ws):
        T.twilight_window_attention(c.kv, q, None, None, 4, NONE, 0, *o, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(10):
        for s, q, o, w in zip(streams, qs, both, ws):
            with torch.cuda.stream(s):
                T.twilight_window_attention(c.kv, q, None, None, 4, NONE, 0, *o, w)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_without_lse_and_default_rows():
    import paper_2502_02770_amd as T
    c = Cache([100, 700], 8, 2, seed=16)
    q = queries(2 * 6, 8, 1)
    a, lse = sent(q, 8)
    T.twilight_window_attention(c.kv, q, None, None, 6, 50, 3, a, lse, workspace(c.kv, 6))
    b = torch.zeros_like(a)
    T.twilight_window_attention(c.kv, q, i32([6, 6]), i32([0, 6]), 6, 50, 3, b, None, workspace(c.kv, 6))
    assert torch.equal(a, b)


def test_one_token_equals_the_dense_decode():
    """max_new = 1 with everything visible is twilight_sparse_decode over all tokens."""
    import paper_2502_02770_amd as T
    c = Cache([5, 3000, 177], 32, 8, seed=17)
    q = queries(3, 32, 2)
    dense, dl = torch.empty_like(q), torch.empty(3, 32, device="cuda")
    ws = torch.empty(T.twilight_workspace_bytes(T.TW_WS_DECODE, c.kv, 0, 0), dtype=torch.uint8, device="cuda")
    T.twilight_sparse_decode(c.kv, q, None, None, 0, dense, dl, ws)
    out, lse = sent(q, 32)
    T.twilight_window_attention(c.kv, q, None, None, 1, NONE, 0, out, lse, workspace(c.kv, 1))
    tree, tl = sent(q, 32)
    T.twilight_tree_attention(c.kv, q, None, None, 1, i32([[1], [1], [1]]), 1, tree, tl, workspace(c.kv, 1))
    assert torch.equal(out, tree)
    # both within half a bf16 step (and the weights' rounding, 2^-8 of the values' spread) of the same numbers
    assert (out.float() - dense.float()).abs().max() <= 2.0**-8 * (2 * dense.float().abs().max() + 4.0)
    assert (lse - dl).abs().max() <= 1e-4 and (tl - dl).abs().max() <= 1e-4


def test_results_do_not_depend_on_the_run():
    """Twice the same bits; on another stream; captured and replayed, two graphs over one workspace."""
    import paper_2502_02770_amd as T
    c = Cache([3000, 10, 900], 32, 8, seed=18)
    q, q2 = queries(3 * 12, 32, 3), queries(3 * 12, 32, 4)
    ws = workspace(c.kv, 12)
    mask = i32([[(1 << j % 12) | 1] for j in range(36)])

    def tree(q):
        out, lse = sent(q, 32)
        T.twilight_tree_attention(c.kv, q, None, None, 12, mask, 1, out, lse, ws)
        return out, lse

    def win(q):
        out, lse = sent(q, 32)
        T.twilight_window_attention(c.kv, q, None, None, 12, 300, 7, out, lse, ws)
        return out, lse

    want = [tree(q), win(q), tree(q2), win(q2)]
    for a, b in zip(want, [tree(q), win(q), tree(q2), win(q2)]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = tree(q)
    side.synchronize()
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[0][1])
    qs, graphs = [q.clone(), q.clone()], []
    for f, x in ((tree, qs[0]), (win, qs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = f(x)
        graphs.append((g, o))
    for turn in range(3):
        for k in (0, 1):
            qs[k].copy_(q if turn % 2 == 0 else q2)
        for k in (0, 1):
            graphs[k][0].replay()
        tree(q2)                                                   # eager work in between, on the same workspace
        torch.cuda.synchronize()
        for k in (0, 1):
            w = want[k if turn % 2 == 0 else 2 + k]
            assert torch.equal(graphs[k][1][0], w[0]) and torch.equal(graphs[k][1][1], w[1])
