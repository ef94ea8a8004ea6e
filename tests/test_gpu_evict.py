"""Accumulated attention weights and the choice of the tokens to keep, against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.kv4_util import Cache4, values
from tests.test_gpu_new_tokens import Cache, i32, layout, queries

pytestmark = pytest.mark.gpu
NONE = 2**31 - 1


def _k64(c, b, h):
    """(K rows, magnitudes that a score's error scales with) of a sequence's head, float64."""
    if isinstance(c, Cache4):
        sc, ze = c.bands(b, h)
        return c.rows(0, b, h), 271 * sc + ze
    k = torch.nan_to_num(c.logical[b][0][:, h].double())
    return k, k.abs()


def _see(c, b, m, window, sinks, gone=()):
    n = c.lens[b]
    t, p = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
    s = (t <= p) & ((p - t < window) | (t < sinks))
    for x in gone:
        if x < n:
            s[:, x] = False
    return s


def mass_reference(c, b, q, lse, see):
    """-> (sums [len], their bound).  A score is off by 130 half-steps of its terms' magnitudes (48 of the larger ones of codes, fewer
    than 130), times log2(e)/sqrt(128), a constant off by half a step, as is the product with lse; exp2 and the fma a few steps more, of the
    exponents' size: a relative e of the weight.  Then sums of as many terms as there are rows, in fp32."""
    G, n, m = c.hq // c.hkv, c.lens[b], q.shape[0]
    got, bound = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    for h in range(c.hq):
        k, mags = _k64(c, b, h // G)
        x = (q[:, h].double() @ k.T) / math.sqrt(128)
        mag = (q[:, h].double().abs() @ mags.T) / math.sqrt(128)
        l = lse[:, h].double()
        ok = torch.isfinite(l)
        l = torch.where(ok, l, torch.zeros_like(l))[:, None]
        w = torch.where(see & ok[:, None], torch.exp(x - l), torch.zeros_like(x))
        e = 130 * 2.0**-24 * mag + 4 * 2.0**-24 * (x.abs() + l.abs()) + 8 * 2.0**-24
        got += w.sum(0)
        bound += (w * 2 * e).sum(0)
    return got, bound + (m * c.hq + 8) * 2.0**-24 * got


def weigh(c, many, max_new, window=NONE, sinks=0, decay=1.0, seed=0, gap=0, counted=True, gone=None, in_place=False, spread=2.0):
    """Runs twilight_attention_mass on the lse of the definition, and checks it."""
    import paper_2502_02770_amd as T
    off, rows = layout(many, gap)
    q = queries(rows, c.hq, seed, spread)
    lse = torch.full((rows, c.hq), math.nan, device="cuda")
    gone, G = gone or {}, c.hq // c.hkv
    for b, m in enumerate(many):
        see = _see(c, b, m, window, sinks, gone.get(b, ()))
        for h in range(c.hq):
            if m and c.lens[b]:
                x = (q[off[b]:off[b] + m, h].double() @ _k64(c, b, h // G)[0].T) / math.sqrt(128)
                lse[off[b]:off[b] + m, h] = torch.logsumexp(torch.where(see, x, torch.full_like(x, -math.inf)), 1).float()
    g = torch.Generator("cuda").manual_seed(seed)
    before = torch.rand(len(many), c.max_pages * 16, device="cuda", generator=g)
    had, out = before.clone(), torch.full_like(before, 7.0)
    if in_place:
        out = had
    T.twilight_attention_mass(c.kv, q, lse, i32(many) if counted else None, i32(off) if counted else None, max_new, window, sinks, decay, had, out)
    for b, (n, m) in enumerate(zip(c.lens, many)):
        assert torch.equal(out[b, n:], (before if in_place else torch.full_like(before, 7.0))[b, n:])        # positions that are no tokens
        if n == 0:
            continue
        want, bound = mass_reference(c, b, q[off[b]:off[b] + m], lse[off[b]:off[b] + m], _see(c, b, m, window, sinks, gone.get(b, ())))
        old = float(np.float32(decay)) * before[b, :n].double()
        old[max(0, n - m):] = 0
        err = (out[b, :n].double() - want - old).abs()
        assert (err <= bound + 3 * 2.0**-24 * (old + want)).all(), (b, (err - bound).max().item())
    return q, lse, before, out


KIND = pytest.mark.parametrize("kind", [Cache, Cache4])


@KIND
@pytest.mark.parametrize("hq,hkv", [(8, 8), (8, 4), (32, 8), (16, 2), (8, 1), (3, 3)])
@pytest.mark.parametrize("n", [1, 16, 17, 333, 1040])
def test_mass_of_one_token(kind, hq, hkv, n):
    weigh(kind([n], hq, hkv, seed=n), [1], 1, seed=n, counted=False)


@KIND
@pytest.mark.parametrize("window,sinks", [(NONE, 0), (1, 0), (16, 3), (100, 17), (250, 64)])
@pytest.mark.parametrize("new", [2, 5, 33, 130])
def test_mass_of_several(kind, new, window, sinks):
    lens = [400, 1, 177, 2000]
    weigh(kind(lens, 16, 4, seed=new), [min(new, n) for n in lens], new, window, sinks, 0.75, seed=sinks, gap=1)


@KIND
def test_mass_in_place_of_empty_and_shared(kind):
    weigh(kind([0, 5, 700], 8, 2, max_pages=60), [0, 5, 0], 5, decay=0.5, in_place=True)
    weigh(kind([0, 5, 700], 8, 2, max_pages=60), [1, 1, 1], 1, decay=0.0)


@KIND
def test_mass_of_more_new_tokens_than_there_are(kind):
    weigh(kind([4, 90], 8, 2), [9, 9], 9)


@KIND
def test_mass_of_tokens_on_missing_pages(kind):
    c = kind([100, 40], 8, 2)
    gone = {0: set(range(16, 32)) | set(range(96, 112)), 1: set(range(0, 16))}
    for b, p, v in ((0, 1, -1), (0, 6, 1 << 30), (1, 0, -7)):
        c.unmap(b, p, v)
    q, lse, before, out = weigh(c, [2, 2], 2, gone=gone)
    assert torch.equal(out[0, 16:32], before[0, 16:32]) and torch.equal(out[1, :16], before[1, :16])      # (decay 1)


@KIND
def test_rows_without_a_finite_lse_add_nothing(kind):
    import paper_2502_02770_amd as T
    c = kind([200], 8, 2)
    q, lse, before, out = weigh(c, [3], 3)
    lse[0, 1], lse[1, 4], lse[2, 7] = math.nan, math.inf, -math.inf
    got = torch.zeros_like(before)
    T.twilight_attention_mass(c.kv, q, lse, None, None, 3, NONE, 0, 1.0, before, got)
    want, bound = mass_reference(c, 0, q, lse, _see(c, 0, 3, NONE, 0))
    old = before[0, :200].double()
    old[197:] = 0
    assert ((got[0, :200].double() - want - old).abs() <= bound + 3 * 2.0**-24 * (old + want)).all()


@KIND
def test_mass_adds_up_and_repeats_bit_for_bit(kind):
    """All weights of a row are 1 together; no order of waves shows."""
    import paper_2502_02770_amd as T
    c = kind([3000, 50], 32, 8)
    q, lse, before, out = weigh(c, [4, 4], 4, seed=1)
    zero = torch.zeros_like(before)
    got = torch.zeros_like(before)
    T.twilight_attention_mass(c.kv, q, lse, None, None, 4, NONE, 0, 1.0, zero, got)
    assert ((got.double().sum(1) / (4 * 32) - 1).abs() < 1e-4).all()
    for _ in range(3):
        again = torch.zeros_like(before)
        T.twilight_attention_mass(c.kv, q, lse, None, None, 4, NONE, 0, 1.0, zero, again)
        assert torch.equal(again, got)


def test_mass_of_long_context():
    weigh(Cache4([70000, 3], 8, 2, seed=3), [1, 1], 1)
    weigh(Cache([30000], 8, 1, seed=4), [20], 20, 20000, 10)


@KIND
@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8), (8, 1), (10, 5)])
@pytest.mark.parametrize("new,window,sinks", [(17, NONE, 0), (33, 40, 70), (95, 200, 5), (200, NONE, 0)])
def test_mass_of_several_over_many_pages(kind, hq, hkv, new, window, sinks):
    """Four pages to a workgroup: rows in blocks of 16 and 32, the last ones short, and lengths that end inside the four."""
    lens = [5003, 0, 31, 4080]
    weigh(kind(lens, hq, hkv, seed=new), [min(new, n) - (b == 3) for b, n in enumerate(lens)], new, window, sinks, 0.5, seed=hq, gap=2)
    lens = [2993, 405, 3000]                     # (two pages to a workgroup)
    weigh(kind(lens, hq, hkv, seed=new), [new, new - 1, 1], new, window, sinks, 0.5, seed=hq)
    lens = [1701, 333]                           # (one)
    weigh(kind(lens, hq, hkv, seed=new), [new, new // 2], new, window, sinks, 0.5, seed=hq)


@KIND
def test_mass_of_few_over_many_pages(kind):
    for hq, hkv, many, window, sinks in ((8, 8, [9, 3], NONE, 0), (6, 3, [1, 8], 100, 30), (64, 16, [4, 4], 3000, 0), (8, 1, [2, 0], 7, 7000)):
        weigh(kind([6001, 4095], hq, hkv, seed=hkv), many, max(many), window, sinks, 1.0, seed=hkv)
        weigh(kind([6001, 4095], hq, hkv, seed=hkv, max_pages=600), many, max(many), window, sinks, 1.0, seed=hkv)


# -------------------------------------------------------------------------------------------------------------- what to keep
def keep_reference(mass, n, budget, sinks, recent, stride):
    k = max(0, min(budget, n, stride))
    first = min(sinks, k)
    last = min(recent, k - first)
    mid = np.arange(first, n - last)
    key = mass[first:n - last].astype(np.float64)
    key = np.where(np.isnan(key), -np.inf, key)
    worse = np.isnan(mass[first:n - last])                         # behind minus infinity
    best = mid[np.lexsort((mid, -key, worse))][:k - first - last]
    return np.sort(np.concatenate([np.arange(first), best, np.arange(n - last, n)])).astype(np.int32)


def pick(mass, lens, budget, sinks=0, recent=0, stride=None, with_mass=True, max_pages=None):
    import paper_2502_02770_amd as T
    B, L = mass.shape
    assert L % 16 == 0
    stride = stride or max(1, max(budget))
    seq, table = i32(lens), torch.zeros(B, L // 16, dtype=torch.int32, device="cuda")
    kv = T.make_kv(B, 8, 2, L // 16, 4, table, seq)
    idx = torch.full((B, stride), -9, dtype=torch.int32, device="cuda")
    count = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    packed = torch.full((B, stride), 7.0, device="cuda")
    ws = torch.empty(T.twilight_workspace_bytes(T.TW_WS_KEEP, kv), dtype=torch.uint8, device="cuda").fill_(255)
    m = torch.from_numpy(mass).cuda()
    T.twilight_keep_tokens(kv, m, i32(budget), sinks, recent, idx, count, stride, packed if with_mass else None, ws)
    got, counts, pk = idx.cpu().numpy(), count.cpu().numpy(), packed.cpu().numpy()
    for b in range(B):
        want = keep_reference(mass[b], lens[b], budget[b], sinks, recent, stride)
        assert counts[b] == len(want), (b, counts[b], len(want))
        assert np.array_equal(got[b, :len(want)], want), (b, np.flatnonzero(got[b, :len(want)] != want)[:5])
        assert (got[b, len(want):] == -9).all()
        if with_mass:
            assert np.array_equal(pk[b, :len(want)].view(np.int32), mass[b][want].view(np.int32)) and (pk[b, len(want):] == 7.0).all()


def weights(B, L, seed, zeros=0.1):
    rng = np.random.default_rng(seed)
    m = np.exp(2.5 * rng.standard_normal((B, L)) - 4).astype(np.float32)
    m[rng.random((B, L)) < zeros] = 0.0
    return m


# below, at and above what a workgroup takes with 2, 8 and 32 tokens per thread, and rows cut into chunks
SIZES = [1, 15, 16, 100, 2047, 2048, 2049, 8192, 8193, 20000, 32768, 32769, 40960, 40961, 100000]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("share", [0.0, 0.03, 0.5, 0.999, 1.0])
def test_keep_by_size(n, share):
    L = -(-n // 16) * 16
    lens = [n, max(0, n - 1), n // 2, min(n, 7)]
    pick(weights(4, L, n), lens, [max(0, int(share * x)) for x in lens], sinks=2, recent=3, stride=L)


@pytest.mark.parametrize("n", [300, 5000, 30000, 70000])
def test_keep_of_equal_weights(n):
    """Equal ones from the lowest position up; a few larger ones among them."""
    L = -(-n // 16) * 16
    m = np.full((3, L), 0.25, dtype=np.float32)
    m[1, ::7] = 0.5
    m[2] = np.where(np.arange(L) % 3 == 0, 0.0, -0.0).astype(np.float32)
    pick(m, [n, n - 3, n], [n // 3, n // 4, n // 2], sinks=4, recent=10)


@pytest.mark.parametrize("n", [200, 40000])
def test_keep_of_any_numbers(n):
    """Negative ones, infinities, the smallest; what is no number last."""
    L = -(-n // 16) * 16
    rng = np.random.default_rng(n)
    m = rng.standard_normal((2, L)).astype(np.float32)
    for v in (math.inf, -math.inf, math.nan, -math.nan, 1e-45, -1e-45, 0.0, -0.0, 3.4e38, -3.4e38):
        m[rng.random((2, L)) < 0.02] = v
    pick(m, [n, n - 5], [n // 2, n - 6])
    pick(m, [n, n - 5], [n - 1, n // 9], sinks=1, recent=1)
    m[:] = math.nan
    pick(m, [n, n - 5], [n // 2, n - 6], sinks=3)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (5, 0), (0, 5), (4, 100), (100, 4), (1000, 1000), (NONE, 0), (0, NONE)])
@pytest.mark.parametrize("n", [64, 1000, 36000])
def test_keep_of_first_and_latest(n, sinks, recent):
    L = -(-n // 16) * 16
    for budget in ([0, 1, 3], [7, 50, 101], [n, n + 5, 2**31 - 1], [-1, -2**31, n - 1]):
        pick(weights(3, L, n), [n, n, n - 9], budget, sinks, recent, stride=L)


def test_keep_writes_no_more_than_its_rows():
    pick(weights(3, 4096, 0), [4000, 4096, 17], [3000, 10, 3000], 4, 8, stride=100)
    pick(weights(2, 50000, 0), [50000, 33333], [3000, 10], 4, 8, stride=1111, with_mass=False)


def test_keep_of_a_very_long_row():
    """More than 128 x 8192 tokens: chunks of two blocks."""
    n = 1_100_003
    L = -(-n // 16) * 16
    m = np.concatenate([weights(1, L, 5), np.round(weights(1, L, 6), 2).astype(np.float32)])
    pick(m, [n, n - 70000], [n // 3, n // 5], 16, 4096)


def test_keep_of_a_batch():
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 3000, 100)]
    pick(weights(100, 3008, 8), lens, [int(rng.integers(0, x + 2)) for x in lens], 3, 20)


# ------------------------------------------------------------------------------------------------------------ a run of them
@pytest.mark.parametrize("four_bits", [False, True])
def test_steps_with_tokens_given_up(four_bits):
    """A layer's cache that is cut down whenever it passes its budget: every step's attention is that over the tokens still there,
    the weights add up over the steps, the pages behind go back to the pool, and the same in a captured graph."""
    import paper_2502_02770_amd as T
    B, hq, hkv, pages = 2, 8, 2, 8
    table = torch.full((B, pages), -1, dtype=torch.int32)
    make = T.PagedKV4 if four_bits else T.PagedKV
    cache = make(hq, hkv, table, torch.zeros(B, dtype=torch.int32), 30)
    pool, mass = T.PagePool(cache), T.TokenMass(cache)
    g = torch.Generator("cuda").manual_seed(1)
    rand = lambda n, h: torch.randn(n, h, 128, device="cuda", generator=g).to(torch.bfloat16)
    rows = [[], []]                                                # (K, V) of the tokens still there, float64, per sequence
    have = [np.zeros(0), np.zeros(0)]                              # their weight
    lens = [0, 0]
    G = hq // hkv
    for step, many in enumerate([[90, 40]] + [[1, 1]] * 12):
        m = max(many)
        off = [0, m]
        pool.reserve(i32(many), m)
        k, v, q = rand(2 * m, hkv), rand(2 * m, hkv), rand(2 * m, hq) * 3
        cache.append(k, v, cache.seq_lens.clone(), i32(many), i32(off), m)
        cache.seq_lens.add_(i32(many))
        at = T.NewTokens(cache, m)
        out = at.window(q, NONE, 0, i32(many))
        mass.add(q, at.lse, m, n_new=i32(many), decay=0.9)
        lens = [n + x for n, x in zip(lens, many)]
        for b in range(B):
            for i in range(many[b]):
                if four_bits:                                      # what the codes stand for
                    t = lens[b] - many[b] + i
                    p = cache.page_table[b, t // 16].item()
                    kv = [values(x[p, :, t % 16], y[p, :, t % 16]) for x, y in ((cache.kq_pool, cache.kq_meta), (cache.vq_pool, cache.vq_meta))]
                    band = cache.kq_meta[p, :, t % 16].double().abs().repeat_interleave(32, 1)
                    rows[b].append((kv[0], kv[1], 271 * band[..., 0] + band[..., 1]))
                else:
                    rows[b].append((k[off[b] + i].double(), v[off[b] + i].double(), k[off[b] + i].double().abs()))
            K, V, M = (torch.stack([x[j] for x in rows[b]]) for j in range(3))
            n, x = lens[b], many[b]
            new, slack = np.zeros(n), np.zeros(n)
            see = torch.arange(n, device="cuda") <= torch.arange(n - x, n, device="cuda")[:, None]
            for h in range(hq):
                s = (q[off[b]:off[b] + x, h].double() @ K[:, h // G].T) / math.sqrt(128)
                w = torch.softmax(torch.where(see, s, torch.full_like(s, -math.inf)), 1)
                o = w @ V[:, h // G]
                # a score off by e (130 half-steps of its terms' magnitudes and a few of its own), lse by that and the sum's; weights
                # rounded to bf16 or fp16, V to fp16 (2^-8 or 2^-11 + 2^-11 of each), the output to bf16
                e = 130 * 2.0**-24 * (q[off[b]:off[b] + x, h].double().abs() @ M[:, h // G].T).amax(1) / math.sqrt(128) + 2.0**-16
                tol = 2.0**-8 * o.abs() + (2.0**-8 + 2 * e + 400 * 2.0**-24)[:, None] * (w @ V[:, h // G].abs()) + 2.0**-24
                assert ((out[off[b]:off[b] + x, h].double() - o).abs() <= tol).all(), (step, b, h)
                new += w.sum(0).cpu().numpy()
                slack += (w * (3 * e)[:, None]).sum(0).cpu().numpy()
            old = np.concatenate([0.9 * have[b], np.zeros(x)])
            have[b] = old + new
            got = mass.mass[b, :n].double().cpu().numpy()
            assert (np.abs(got - have[b]) <= slack + 2.0**-16 * have[b]).all(), (step, b)        # (fp32 sums of up to 720 weights)
            have[b] = got
        if max(lens) > 64:
            before = [i32([-(-n // 16) for n in lens])]
            kept = mass.evict(i32([50, 30]), num_sinks=2, num_recent=8)
            pool.free((cache.seq_lens + 15) // 16, before[0])
            assert kept.tolist() == [50, 30] and cache.seq_lens.tolist() == [50, 30]
            for b, budget in enumerate((50, 30)):
                want = keep_reference(have[b].astype(np.float32), lens[b], budget, 2, 8, 10**6)
                assert np.array_equal(mass.keep_idx[b, :budget].cpu().numpy(), want)
                rows[b] = [rows[b][t] for t in want]
                have[b] = have[b][want]
                assert np.array_equal(mass.mass[b, :budget].cpu().numpy(), have[b].astype(np.float32))
            lens = [50, 30]
            assert int((pool.ref_count > 0).sum()) == 4 + 2 and (cache.page_table >= 0).sum().item() == 6
    assert lens[0] > 50 and pool.status.item() == 0


def test_a_captured_step_of_mass_and_choice():
    """Attention, weights, choice and compaction in one graph, replayed with eager work between: as run eagerly."""
    import paper_2502_02770_amd as T
    hq, hkv, B, pages = 8, 2, 2, 20

    def build():
        table = torch.arange(B * pages, dtype=torch.int32).view(B, pages)
        cache = T.PagedKV4(hq, hkv, table, torch.tensor([300, 77], dtype=torch.int32), B * pages)
        g = torch.Generator("cuda").manual_seed(5)
        k, v = (torch.randn(600, hkv, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        cache.append(k, v, i32([0, 0]), i32([300, 300]), i32([0, 300]), 300)
        return cache, T.NewTokens(cache, 1), T.TokenMass(cache)

    def step(cache, at, mass, q, budget):
        at.window(q, NONE, 0)
        mass.add(q, at.lse, 1)
        mass.evict(budget, 2, 4)

    q, budget = queries(2, hq, 3), i32([300, 77])
    eager, captured = build(), build()
    cache, at, mass = captured
    for x in (eager, captured):
        step(*x, q, budget)                                        # (nothing given up yet)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, at, mass, q, budget)
    for n in ((250, 70), (200, 70), (120, 33), (16, 1)):
        budget.copy_(i32(list(n)))
        q.copy_(queries(2, hq, sum(n)))
        graph.replay()
        step(*eager, q, budget)
        torch.cuda.synchronize()
        assert torch.equal(at.out, eager[1].out) and torch.equal(mass.mass, eager[2].mass) and cache.seq_lens.tolist() == list(n)
        assert torch.equal(cache.seq_lens, eager[0].seq_lens) and torch.equal(cache.kq_pool, eager[0].kq_pool)
        assert torch.equal(cache.vq_meta.view(torch.int16), eager[0].vq_meta.view(torch.int16))


def test_a_cache_with_bounds_in_four_bits_is_not_cut_down():
    """The codes do not give the rows' bounds back: refused before anything moves."""
    import paper_2502_02770_amd as T
    cache = T.PagedKV4(8, 2, torch.arange(4, dtype=torch.int32).view(1, 4), torch.tensor([50], dtype=torch.int32), 4, with_bounds=True)
    x = queries(50, 2, 1)
    cache.append(x, x, i32([0]), i32([50]), i32([0]), 50)
    mass = T.TokenMass(cache)
    had = [t.clone() for t in (cache.kq_pool, cache.vq_pool, cache.page_minmax, mass.mass)]
    with pytest.raises(RuntimeError):
        mass.evict(i32([20]))
    assert all(torch.equal(t, h) for t, h in zip((cache.kq_pool, cache.vq_pool, cache.page_minmax, mass.mass), had)) and cache.seq_lens.tolist() == [50]


def test_two_streams_with_a_workspace_each():
    import paper_2502_02770_amd as T
    L = 40000
    m = torch.from_numpy(weights(2, L, 1)).cuda()
    kv = T.make_kv(2, 8, 2, L // 16, 4, torch.zeros(2, L // 16, dtype=torch.int32, device="cuda"), i32([L, L - 100]))
    seq = i32([L, L - 100])
    kv.seq_lens = seq.data_ptr()
    res = []
    for _ in range(2):
        res.append((torch.cuda.Stream(), torch.zeros(2, 5000, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"),
                    torch.empty(T.twilight_workspace_bytes(T.TW_WS_KEEP, kv), dtype=torch.uint8, device="cuda")))
    budgets = [i32([5000, 3000]), i32([77, 4999])]
    torch.cuda.synchronize()
    for _ in range(5):
        for (s, idx, count, ws), budget in zip(res, budgets):
            with torch.cuda.stream(s):
                T.twilight_keep_tokens(kv, m, budget, 2, 9, idx, count, 5000, None, ws)
    torch.cuda.synchronize()
    for (s, idx, count, ws), budget in zip(res, budgets):
        for b, n in enumerate((L, L - 100)):
            want = keep_reference(m[b].cpu().numpy(), n, budget[b].item(), 2, 9, 5000)
            assert count[b].item() == len(want) and np.array_equal(idx[b, :len(want)].cpu().numpy(), want)
