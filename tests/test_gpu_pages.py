"""Pages of the cache: handed out, shared, given back, copied, compacted - against plain sequential Python - and a speculative
step, a streaming step and beams made of them together with the operators that were there."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32)).cuda()


class Model:
    """The documented behaviour, one entry at a time."""

    def __init__(self, table, lens, pool):
        self.table, self.lens, self.pool = np.array(table), list(lens), pool
        self.ref = np.zeros(pool, dtype=np.int64)
        for p in self.table.reshape(-1):
            if 0 <= p < pool:
                self.ref[p] += 1
        self.status = 0

    def take(self):
        free = np.flatnonzero(self.ref == 0)
        if not len(free):
            self.status |= 4
            return -1
        self.ref[free[0]] = 1
        return int(free[0])

    def drop(self, p):
        if self.ref[p] <= 0:
            self.status |= 8
        else:
            self.ref[p] -= 1

    def reserve(self, n_new, max_new):
        MP = self.table.shape[1]
        for b, n in enumerate(n_new):
            n = max(0, min(n, max_new))
            if n:
                for p in range(self.lens[b] // 16, min(MP, -(-(self.lens[b] + n) // 16))):
                    if not 0 <= self.table[b, p] < self.pool:
                        self.table[b, p] = self.take()

    def free(self, first, end):
        for b in range(len(self.lens)):
            for p in range(max(first[b], 0), min(end[b], self.table.shape[1])):
                if 0 <= self.table[b, p] < self.pool:
                    self.drop(self.table[b, p])
                    self.table[b, p] = -1

    def fork(self, parent):
        MP = self.table.shape[1]
        new = np.full((len(parent), MP), -1, dtype=np.int32)
        lens, src, dst, asked = [], [], [], []
        children = [0] * len(self.lens)
        for i, r in enumerate(parent):
            src.append(-1)
            dst.append(-1)
            if not 0 <= r < len(self.lens):
                lens.append(0)
                continue
            lens.append(self.lens[r])
            children[r] += 1
            full = self.lens[r] // 16
            for p in range(MP):
                if 0 <= self.table[r, p] < self.pool and (p < full or children[r] == 1):
                    new[i, p] = self.table[r, p]
            if children[r] > 1 and self.lens[r] % 16 and 0 <= self.table[r, full] < self.pool:
                asked.append((i, full, self.table[r, full]))
        for r, c in enumerate(children):
            full = self.lens[r] // 16
            for p in range(MP):
                if 0 <= self.table[r, p] < self.pool:
                    if c == 0:
                        self.drop(self.table[r, p])
                    elif p < full:
                        self.ref[self.table[r, p]] += c - 1
        for i, p, s in asked:
            got = self.take()
            if got >= 0:
                new[i, p], src[i], dst[i] = got, s, got
        self.table, self.lens = new, lens
        return src, dst


def cache_of(table, lens, pool, hq=8, hkv=2, bits=4, fill=True, seed=0):
    import paper_2502_02770_amd as T
    c = T.PagedKV(hq, hkv, torch.from_numpy(np.array(table, dtype=np.int32)), torch.tensor(lens, dtype=torch.int32), pool, "cuda", quant_bits=bits)
    if fill:
        g = torch.Generator("cuda").manual_seed(seed)
        c.k_pool.normal_(generator=g)
        c.v_pool.normal_(generator=g)
        c.kq_pool.random_(0, 256, generator=g)
        c.kq_meta.normal_(generator=g)
        c.page_minmax.normal_(generator=g)
    return c


@pytest.mark.parametrize("batch,max_pages,pool,seed", [(1, 1, 1, 0), (3, 7, 12, 1), (9, 40, 300, 2), (70, 33, 2000, 3), (17, 600, 40000, 4), (1100, 5, 5000, 5), (5000, 3, 9000, 6)])
def test_random_life_of_a_pool(batch, max_pages, pool, seed):
    import paper_2502_02770_amd as T
    rng = np.random.default_rng(seed)
    table = np.full((batch, max_pages), -1, dtype=np.int32)
    if seed % 2:                                                   # unmapped is whatever lies outside the pool
        table[:] = rng.choice([-1, -7, pool, 2**31 - 1], table.shape)
    m = Model(table, [0] * batch, pool)
    c = cache_of(table, [0] * batch, pool, fill=False)
    pp = T.PagePool(c)
    for step in range(12):
        do = rng.choice(["reserve", "reserve", "free", "fork"])
        if do == "reserve":
            most = int(rng.integers(1, 16 * max_pages + 40))
            n = rng.integers(-2, most + 1, batch) * (rng.random(batch) < 0.7)
            m.reserve(n.tolist(), most)
            pp.reserve(i32(n), most)
            grown = [min(x + max(0, int(y)), max_pages * 16) if rng.random() < 0.8 else x for x, y in zip(m.lens, n)]
            m.lens = grown
        elif do == "free":
            first = rng.integers(-3, max_pages + 1, batch)
            end = first + rng.integers(-2, max_pages + 2, batch) * (rng.random(batch) < 0.5)
            m.free(first.tolist(), end.tolist())
            pp.free(i32(first), i32(end))
        else:
            parent = np.where(rng.random(batch) < 0.5, np.arange(batch), rng.integers(-1, batch + 1, batch))
            src, dst = m.fork(parent.tolist())
            t, l, s, d = pp.fork(i32(parent))
            assert l.tolist() == m.lens and s.tolist() == src and d.tolist() == dst, (step, do)
            c.page_table.copy_(t)
        assert np.array_equal(c.page_table.cpu().numpy()[m.table >= 0], m.table[m.table >= 0]), (step, do)
        got = c.page_table.cpu().numpy()
        assert np.array_equal((got >= 0) & (got < pool), (m.table >= 0) & (m.table < pool)), (step, do)
        assert np.array_equal(pp.ref_count.cpu().numpy(), m.ref), (step, do)
        assert int(pp.status) == m.status, (step, do)
        c.seq_lens.copy_(i32(m.lens))


def test_fork_into_larger_and_smaller_batches():
    import paper_2502_02770_amd as T
    table = np.arange(3 * 6, dtype=np.int32).reshape(3, 6)
    lens = [33, 96, 5]
    for parent in ([0] * 5, [2, 2, 0, 1, 1, -1, 0], [1], [-1, 9]):
        m, c = Model(table, lens, 40), cache_of(table, lens, 40, fill=False)
        pp = T.PagePool(c)
        src, dst = m.fork(parent)
        t, l, s, d = pp.fork(i32(parent))
        assert t.cpu().numpy().tolist() == m.table.tolist() and l.tolist() == m.lens
        assert s.tolist() == src and d.tolist() == dst and np.array_equal(pp.ref_count.cpu().numpy(), m.ref)


def test_references_given_back_twice_are_reported():
    import paper_2502_02770_amd as T
    c = cache_of([[3, 4], [3, 5]], [32, 32], 8, fill=False)
    pp = T.PagePool(c)
    pp.ref_count[3] = 1                                            # one count short
    pp.free(i32([0, 0]), i32([2, 2]))
    assert pp.ref_count.tolist() == [0] * 8 and int(pp.status) == 8 and (c.page_table == -1).all()


POOLS = ("k_pool", "v_pool", "kq_pool", "kq_meta", "page_minmax")


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("hkv", [1, 8])
def test_copied_pages(bits, hkv):
    c = cache_of([[0]], [1], 50, hkv, hkv, bits)
    before = {n: getattr(c, n).clone() for n in POOLS}
    src, dst = [3, 7, -1, 9, 7, 50, 2, 11], [10, 0, 20, 9, 49, 21, -1, 2**31 - 1]
    c.copy_pages(i32(src), i32(dst))
    for s, d in ((3, 10), (7, 0), (7, 49)):
        for n in POOLS:
            before[n][d] = before[n][s]
    for n in POOLS:
        assert torch.equal(getattr(c, n).view(torch.uint8), before[n].view(torch.uint8)), n


def test_more_copies_than_32_bits_count():
    """2^31 (pair, KV head) items, all but two of them passed over."""
    c = cache_of([[0]], [1], 5, 8, 8)
    src = torch.full((1 << 28,), -1, dtype=torch.int32, device="cuda")
    dst = src.clone()
    src[[0, -1]], dst[[0, -1]] = i32([3, 1]), i32([0, 4])
    before = {n: getattr(c, n).clone() for n in POOLS}
    c.copy_pages(src, dst)
    for n in POOLS:
        before[n][0], before[n][4] = before[n][3], before[n][1]
        assert torch.equal(getattr(c, n).view(torch.uint8), before[n].view(torch.uint8)), n


def test_a_reservation_of_any_number_is_clipped_to_the_row():
    c = cache_of([[-1] * 6, [-1] * 6], [0, 17], 20)
    import paper_2502_02770_amd as T
    pp = T.PagePool(c)
    pp.reserve(i32([2**31 - 1, 2**31 - 1]), 2**31 - 1)
    assert c.page_table.tolist() == [[0, 1, 2, 3, 4, 5], [-1, 6, 7, 8, 9, 10]] and int(pp.status) == 0


def compact_model(c, keep, count, start, to):
    """-> pools after, and the bounds' pages that are taken again {(page): rows valid}"""
    p = {n: getattr(c, n).clone().cpu() for n in POOLS}
    old = {n: x.clone() for n, x in p.items()}
    table, lens, MP = c.page_table.cpu().numpy(), c.seq_lens.cpu().tolist(), c.max_pages
    for b in range(c.batch):
        n = max(0, min(count[b], keep.shape[1]))
        for i in range(n):
            t, d = int(keep[b, i]), start[b] + i
            if not 0 <= t < lens[b] or d >= MP * 16:
                continue
            sp, dp = table[b, t // 16], to[b, d // 16]
            if not (0 <= sp < c.num_pool_pages and 0 <= dp < c.num_pool_pages):
                continue
            for name in POOLS[:4]:
                p[name][dp, :, d % 16] = old[name][sp, :, t % 16]
        end = start[b] + n
        for page in range(start[b] // 16, min(MP, -(-end // 16))):
            dp = to[b, page]
            if 0 <= dp < c.num_pool_pages:
                rows = p["k_pool"][dp, :, :min(16, end - page * 16)]
                p["page_minmax"][dp, :, 0], p["page_minmax"][dp, :, 1] = rows.amin(1), rows.amax(1)
    return p


def check_pools(c, want):
    for n in POOLS:
        got = getattr(c, n).cpu()
        assert torch.equal(got, want[n]) or torch.equal(got.view(torch.uint8), want[n].view(torch.uint8)), n


@pytest.mark.parametrize("bits,hkv", [(4, 8), (2, 1), (8, 3)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compaction(bits, hkv, in_place):
    rng = np.random.default_rng(bits + hkv)
    lens = [1, 16, 40, 700, 333, 129, 64, 1500, 20]
    MP = 100
    table = np.full((len(lens), MP), -1, dtype=np.int32)
    ids = rng.permutation(500)
    at = 0
    for b, n in enumerate(lens):
        h = -(-n // 16)
        table[b, :h] = ids[at:at + h]
        at += h
    to = table
    if not in_place:
        to = np.full_like(table, -1)
        for b, n in enumerate(lens):
            h = -(-n // 16) + 1
            to[b, :h] = ids[at:at + h]
            at += h
    start = [0, 3, 17, 0, 100, 129, 5, 16, 13]
    keeps = []
    for b, n in enumerate(lens):
        pick = np.arange(start[b] if in_place else 0, n)
        pick = np.sort(rng.permutation(pick)[:int(len(pick) * rng.choice([0.3, 0.7, 1.0]))])
        keeps.append(pick)
    keeps[8] = keeps[8][:0]                                        # nothing kept: the page is cut back to its first tokens
    stride = max(len(k) for k in keeps) + 2
    keep = rng.integers(-5, 3000, (len(lens), stride)).astype(np.int32)       # (garbage beyond the counts)
    for b, k in enumerate(keeps):
        keep[b, :len(k)] = k
    count = [len(k) for k in keeps]
    c = cache_of(table, lens, 500, hkv, hkv, bits, seed=bits)
    want = compact_model(c, keep, count, start, to)
    c.compact(i32(keep), i32(count), i32(start), None if in_place else i32(to))
    check_pools(c, want)


def test_compaction_passes_over_what_is_not_there():
    """Positions outside the sequence, sources and destinations on unmapped pages, counts beyond the row, a row at its end."""
    table = np.array([[5, -1, 6, 99], [7, 8, 9, 10]], dtype=np.int32)
    to = np.array([[11, 12, -1, 13], [14, 1000, 15, 16]], dtype=np.int32)
    keep = np.array([[0, 18, 40, -3, 61, 64, 10**9, 3], [1, 2, 3, 4, 5, 6, 7, 60]], dtype=np.int32)
    c = cache_of(table, [62, 61], 30)
    want = compact_model(c, keep, [100, 8], [14, 60], to)
    c.compact(i32(keep), i32([100, 8]), i32([14, 60]), i32(to))
    check_pools(c, want)
    c = cache_of(table, [62, 61], 30)
    want = {n: getattr(c, n).clone().cpu() for n in POOLS}
    c.compact(i32(keep), i32([0, -4]), i32([16, 48]))              # nothing kept, nothing cut
    check_pools(c, want)


def test_compaction_of_a_cache_without_copy_or_values():
    import paper_2502_02770_amd as T
    c = cache_of([[0, 1, 2]], [40], 4)
    kv = T.make_kv(1, 8, 2, 3, 4, c.page_table, c.seq_lens, c.k_pool)
    want = compact_model(c, np.array([[20, 30, 35]]), [3], [18], c.page_table.cpu().numpy())["k_pool"]
    others = {n: getattr(c, n).clone() for n in POOLS[1:]}
    T.twilight_tokens_compact(kv, i32([[20, 30, 35]]), i32([3]), 3, i32([18]), None)
    assert torch.equal(c.k_pool.cpu(), want)
    T.twilight_pages_copy(kv, i32([0]), i32([3]), 1)
    assert torch.equal(c.k_pool[3], c.k_pool[0])
    for n in others:
        assert torch.equal(getattr(c, n).view(torch.uint8), others[n].view(torch.uint8)), n


def rows(n, hkv, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return [torch.randn(n, hkv, 128, device="cuda", dtype=torch.bfloat16, generator=g) for _ in "kv"]


@pytest.mark.parametrize("bits", [4, 8])
def test_a_speculative_step(bits):
    """reserve -> append the draft -> tree attention -> compact the accepted path -> free: the cache that is left is the one to which
    the accepted tokens alone were appended, bit for bit, for the selector and pruner too."""
    import paper_2502_02770_amd as T
    from paper_2502_02770_amd.cache import tree_mask_of_parents
    hq, hkv, B, N = 32, 8, 3, 24
    lens, MP, pool = [70, 16, 301], 24, 80
    rng = np.random.default_rng(0)
    prompt = [rows(n, hkv, 10 + b) for b, n in enumerate(lens)]
    draft = rows(B * N, hkv, 20)
    parents = np.stack([[int(rng.integers(max(-1, j - 3), j)) if j else -1 for j in range(N)] for _ in range(B)])
    mask = tree_mask_of_parents(torch.from_numpy(parents)).reshape(B * N, -1).cuda()
    path = []                                                      # accepted: a chain of the tree
    for b in range(B):
        j, chain = N - 1 - 5 * b, []
        while j >= 0:
            chain.append(j)
            j = int(parents[b, j])
        path.append(chain[::-1])
    zero = i32([0] * B)

    def new_cache():
        c = cache_of(np.full((B, MP), -1), [0] * B, pool, hq, hkv, bits, fill=False)
        p = T.PagePool(c)
        p.reserve(i32(lens), max(lens))
        c.append(torch.cat([x[0] for x in prompt]), torch.cat([x[1] for x in prompt]), zero, i32(lens), i32(np.cumsum([0] + lens[:-1])), max(lens))
        c.seq_lens.copy_(i32(lens))
        return c, p

    c, p = new_cache()
    p.reserve(i32([N] * B), N)
    c.append(draft[0], draft[1], c.seq_lens.clone(), i32([N] * B), i32([b * N for b in range(B)]), N)
    start = c.seq_lens.clone()
    c.seq_lens += N
    st = T.NewTokens(c, N)
    q = torch.randn(B * N, hq, 128, device="cuda").to(torch.bfloat16)
    out = st.tree(q, mask).clone()
    # every accepted token's row is what a decode over its own path gives: the window form over a cache with the path alone
    keep = np.full((B, N), -1, dtype=np.int32)
    for b, chain in enumerate(path):
        keep[b, :len(chain)] = [lens[b] + j for j in chain]
    count = i32([len(x) for x in path])
    c.compact(i32(keep), count, start)
    c.seq_lens.copy_(start + count)
    used = (c.seq_lens + 15) // 16
    p.free(used, torch.full_like(used, MP))
    r, rp = new_cache()                                            # the same without the rejected tokens
    rp.reserve(count, N)
    at = i32(np.cumsum([0] + [len(x) for x in path[:-1]]))
    pick = torch.cat([torch.tensor([b * N + j for j in chain]) for b, chain in enumerate(path)]).cuda()
    r.append(draft[0][pick].contiguous(), draft[1][pick].contiguous(), r.seq_lens.clone(), count, at, N)
    r.seq_lens += count
    for b in range(B):
        n = int(r.seq_lens[b])
        a, z = c.page_table[b, :-(-n // 16)].long(), r.page_table[b, :-(-n // 16)].long()
        for name in POOLS[:4]:
            x, y = (getattr(o, name)[i].transpose(1, 2).flatten(0, 1)[:n] for o, i in ((c, a), (r, z)))
            assert torch.equal(x, y), (b, name)
        assert torch.equal(c.page_minmax[a], r.page_minmax[z]), b
    assert int(p.ref_count.sum()) == int(used.sum()) and int(p.status) == int(rp.status) == 0
    win = T.NewTokens(r, N)
    qw = torch.zeros_like(q)
    for b, chain in enumerate(path):
        qw[b * N:b * N + len(chain)] = q[[b * N + j for j in chain]]
    got = win.window(qw, 2**31 - 1, n_new=count)
    for b, chain in enumerate(path):
        x, y = out[[b * N + j for j in chain]].float(), got[b * N:b * N + len(chain)].float()
        # each side: weights rounded to bf16 (2^-8 of values within 6), the output by half a step
        assert (x - y).abs().max() <= 2 * 2.0**-8 * (6 + x.abs().max())
    res = []
    for o in (c, r):
        s = T.DecodeStep(o, max_sel=6, with_kept_idx=True)
        s.run(q[:B].contiguous(), i32([64] * B), 0.9)
        res.append([s.sel_pages, s.sel_count, s.union_count, s.out, s.lse] + [s.union_idx[g, :int(s.union_count[g])] for g in range(B * hkv)])
    assert all(torch.equal(x, y) for x, y in zip(*res))


def test_a_streaming_step():
    """reserve -> append -> window attention -> free behind the window, token by token over a small pool: the results are those of a
    cache that keeps everything."""
    import paper_2502_02770_amd as T
    hq, hkv, B, W, S = 16, 4, 2, 40, 5
    steps, MP = 150, 10
    small, big = (cache_of(np.full((B, MP), -1), [0] * B, n, hq, hkv, fill=False) for n in (2 * 5, 2 * MP))
    pools = [T.PagePool(x) for x in (small, big)]
    st = [T.NewTokens(x, 1) for x in (small, big)]
    one, at = i32([1] * B), i32(range(B))
    for t in range(steps):
        k, v = rows(B, hkv, t)
        q = torch.randn(B, hq, 128, device="cuda").to(torch.bfloat16)
        got = []
        for x, p, s in zip((small, big), pools, st):
            p.reserve(one, 1)
            x.append(k, v, x.seq_lens.clone(), one, at, 1)
            x.seq_lens += 1
            got.append(s.window(q, W, S).clone())
        assert torch.equal(got[0], got[1]), t
        pools[0].free_behind(W, S)
        assert int(pools[0].status) == 0, t
    assert int((pools[0].ref_count > 0).sum()) <= 2 * 5 < int((pools[1].ref_count > 0).sum())


def test_beams():
    """fork -> copy -> append: every beam attends as if its cache were its own."""
    import paper_2502_02770_amd as T
    hq, hkv, B, MP = 8, 2, 4, 8
    c = cache_of(np.full((B, MP), -1), [0] * B, 40, hq, hkv, fill=False)
    p = T.PagePool(c)
    hist = [[] for _ in range(B)]
    rng = np.random.default_rng(0)
    one, at = i32([1] * B), i32(range(B))
    for t in range(60):
        p.reserve(one, 1)
        k, v = rows(B, hkv, t)
        c.append(k, v, c.seq_lens.clone(), one, at, 1)
        c.seq_lens += 1
        hist = [h + [(t, b)] for b, h in enumerate(hist)]
        if t % 7 == 3:
            parent = rng.integers(0, B, B)
            table, lens, src, dst = p.fork(i32(parent))
            c.copy_pages(src, dst)
            c.page_table.copy_(table)
            c.seq_lens.copy_(lens)
            hist = [hist[r] for r in parent]
    assert int(p.status) == 0
    st = T.NewTokens(c, 1)
    q = torch.randn(B, hq, 128, device="cuda").to(torch.bfloat16)
    out = st.window(q, 2**31 - 1).clone()
    for b in range(B):
        own = cache_of([list(range(MP))], [60], MP, hq, hkv, fill=False)
        kk, vv = (torch.stack([rows(B, hkv, t)[i][r] for t, r in hist[b]]) for i in (0, 1))
        own.append(kk, vv, i32([0]), i32([60]), i32([0]), 60)
        assert torch.equal(T.NewTokens(own, 1).window(q[b:b + 1].contiguous(), 2**31 - 1), out[b:b + 1]), b


def test_samples_of_one_prompt():
    """One row forked into a larger batch over the same pools: full pages shared, the partly filled one copied, each sample going on
    by itself; then the samples but one dropped."""
    import paper_2502_02770_amd as T
    hq, hkv, n, N = 8, 2, 37, 5
    c = cache_of([[-1] * 6], [0], 20, hq, hkv, fill=False)
    p = T.PagePool(c)
    p.reserve(i32([n]), n)
    k, v = rows(n, hkv, 1)
    c.append(k, v, i32([0]), i32([n]), i32([0]), n)
    c.seq_lens += n
    table, lens, src, dst = p.fork(i32([0] * N))
    c.copy_pages(src, dst)
    s = c.over(table, lens)
    ps = p.over(s)
    assert ps.ref_count[table[0, :2].long()].tolist() == [N, N] and len(set(table[:, 2].tolist())) == N
    kn, vn = rows(N, hkv, 2)
    ps.reserve(i32([1] * N), 1)
    s.append(kn, vn, s.seq_lens.clone(), i32([1] * N), i32(range(N)), 1)
    s.seq_lens += 1
    q = torch.randn(N, hq, 128, device="cuda").to(torch.bfloat16)
    out = T.NewTokens(s, 1).window(q, 2**31 - 1).clone()
    for b in range(N):
        own = cache_of([list(range(3))], [n + 1], 3, hq, hkv, fill=False)
        own.append(torch.cat([k, kn[b:b + 1]]), torch.cat([v, vn[b:b + 1]]), i32([0]), i32([n + 1]), i32([0]), n + 1)
        assert torch.equal(T.NewTokens(own, 1).window(q[b:b + 1].contiguous(), 2**31 - 1), out[b:b + 1]), b
    table, lens, src, dst = ps.fork(i32([3]))
    assert lens.tolist() == [n + 1] and src.tolist() == dst.tolist() == [-1]
    assert int((ps.ref_count > 0).sum()) == 3 and int(ps.ref_count.sum()) == 3 and int(ps.status) == 0


def test_pages_captured_and_replayed():
    """reserve, free, fork and compaction hold no host state: a replayed graph does what the calls did."""
    import paper_2502_02770_amd as T
    table, lens, pool = [[0, 1, 2, -1], [3, 4, -1, -1]], [40, 20], 20
    c = cache_of(table, lens, pool, seed=3)
    pp = T.PagePool(c)
    keep, count, start = i32([[33, 35, 39], [17, 18, 19]]), i32([3, 2]), i32([32, 17])
    parent, n_new, first, end = i32([1, 1, 0]), i32([20, 5]), i32([0, 1]), i32([1, 1])
    saved = {n: getattr(c, n).clone() for n in POOLS}
    t0, r0 = c.page_table.clone(), pp.ref_count.clone()

    def work():
        c.compact(keep, count, start)
        pp.reserve(n_new, 20)
        pp.free(first, end)
        return pp.fork(parent)

    def reset():
        c.page_table.copy_(t0)
        pp.ref_count.copy_(r0)
        for n in POOLS:
            getattr(c, n).copy_(saved[n])

    want = [x.clone() for x in work()] + [c.page_table.clone(), pp.ref_count.clone()] + [getattr(c, n).clone() for n in POOLS]
    reset()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = work()
    for _ in range(3):
        reset()
        g.replay()
        torch.cuda.synchronize()
        now = list(got) + [c.page_table, pp.ref_count] + [getattr(c, n) for n in POOLS]
        assert all(torch.equal(x, y) for x, y in zip(now, want))
