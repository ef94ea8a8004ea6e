"""Arguments at the ends of their ranges for the operators on new tokens and on the cache's pages: what needs no GPU."""
import numpy as np
import pytest
import torch


@pytest.mark.parametrize("window", [1, 2, 16, 17, 40, 1000, 2**31 - 1, 2**31, 2**32, 2**32 + 5, 2**40, 2**63 - 1])
@pytest.mark.parametrize("sinks", [0, 1, 16, 33, 2**31 - 1, 2**32 + 1, 2**36])
def test_pages_behind_a_window(window, sinks):
    """Exactly the pages none of whose tokens the next token sees; the entry's definition, one page at a time."""
    from paper_2502_02770_amd.cache import pages_behind
    lens = [0, 1, 15, 16, 64, 100, 1000, 5000]
    first, end = pages_behind(torch.tensor(lens, dtype=torch.int32), window, sinks)
    assert first.dtype == end.dtype == torch.int32 and (first >= 0).all() and (end >= 0).all()
    for n, lo, hi in zip(lens, first.tolist(), end.tolist()):
        unseen = {p for p in range(n // 16) if all(n - t >= window and t >= sinks for t in range(16 * p, 16 * p + 16))}
        assert set(range(lo, hi)) == unseen, n


@pytest.mark.parametrize("window", [2**31 - 1, 2**32, 2**40, 2**63 - 1])
def test_nothing_is_given_back_behind_a_window_without_limit(window):
    import paper_2502_02770_amd as T
    p = object.__new__(T.PagePool)
    p.cache = object.__new__(T.PagedKV)
    p.cache.seq_lens, p.cache.batch, given = torch.tensor([1000, 64], dtype=torch.int32), 2, []
    p.free = lambda first, end: given.append((first.tolist(), end.tolist()))
    p.free_behind(window, 4)
    p.free_behind(40, 2**36)                                       # sinks without limit
    for first, end in given:
        assert all(hi <= lo for lo, hi in zip(first, end)), (first, end)


def test_lengths_outside_a_row_give_back_nothing_by_a_wrap():
    from paper_2502_02770_amd.cache import pages_behind
    lens = torch.tensor([-5, -2**31, 2**31 - 1], dtype=torch.int32)
    assert pages_behind(lens, 2**63 - 1, 0)[1].tolist() == [0, 0, 0]
    assert pages_behind(lens, 1, 0)[1].tolist() == [0, 0, (2**31 - 1) // 16]


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 0), (-2**40, 0), (5, -1), (5, -2**33)])
def test_windows_and_sinks_that_attention_refuses(window, sinks):
    from paper_2502_02770_amd.cache import pages_behind
    with pytest.raises(AssertionError, match="window"):
        pages_behind(torch.tensor([100], dtype=torch.int32), window, sinks)


def ancestors(parents):
    """Bits of a tree's masks, one token and one step towards the root at a time."""
    see = np.zeros((len(parents), -(-len(parents) // 32) * 32), dtype=bool)
    for j in range(len(parents)):
        k = j
        while True:
            see[j, k] = True
            up = int(parents[k])
            if not 0 <= up < k:
                break
            k = up
    return np.packbits(see, axis=1, bitorder="little").view(np.int32)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_parents_that_are_no_earlier_token_stand_for_the_cache(dtype):
    """Beyond the draft, the token itself or a later one, negative: nothing outside the masks is read."""
    from paper_2502_02770_amd.cache import tree_mask_of_parents
    top = torch.iinfo(dtype).max
    p = torch.tensor([[0, 0, 5, 9, 40, 3], [-7, top, -top, 1, 3, 4], [3, 2, 2, 2, 6, 33]], dtype=dtype)
    got = tree_mask_of_parents(p).numpy()
    for b in range(3):
        assert np.array_equal(got[b], ancestors(p[b].tolist())), b


@pytest.mark.parametrize("shape", [(0,), (1,), (2, 0), (2,), (1, 33), (3, 2, 64), (2, 200), (1024,)])
@pytest.mark.parametrize("kind", ["any", "chain", "star"])
def test_masks_of_trees_of_any_depth(shape, kind):
    from paper_2502_02770_amd.cache import tree_mask_of_parents
    n, rng = shape[-1], np.random.default_rng(shape[-1])
    p = np.broadcast_to(np.arange(n) - 1, shape) if kind == "chain" else np.zeros(shape) if kind == "star" else (
        np.floor(rng.random(shape) * (np.arange(n) + 1)) - 1)
    got = tree_mask_of_parents(torch.from_numpy(p.astype(np.int32)))
    assert got.shape == (*shape, -(-n // 32)) and got.dtype == torch.int32 and got.is_contiguous()
    for tree, words in zip(p.reshape(-1, n), got.reshape(-1, n, got.shape[-1]).numpy()) if n else ():
        assert np.array_equal(words, ancestors(tree))


def test_masks_take_steps_of_the_logarithm_of_the_draft():
    """A draft of 128 tokens: operations of torch, each a launch of some microseconds ahead of the attention."""
    from torch.utils._python_dispatch import TorchDispatchMode
    from paper_2502_02770_amd.cache import tree_mask_of_parents

    class Count(TorchDispatchMode):
        n = 0

        def __torch_dispatch__(self, f, types, args=(), kwargs=None):
            Count.n += 1
            return f(*args, **(kwargs or {}))

    with Count():
        tree_mask_of_parents(torch.arange(-1, 127, dtype=torch.int32).expand(4, 128))
    assert Count.n <= 30 + 10 * 7, Count.n                         # per step two look-ups of a few operations each and a union


def _calls(B, n):
    """Every call of the operators on new tokens and pages with n in one of its sizes."""
    ws = torch.zeros(4)
    kv = B.twilight_kv_t()
    t = None
    return {
        "tree max_new": lambda: B.twilight_tree_attention(kv, t, t, t, n, t, 1, t, t, ws),
        "tree mask_words": lambda: B.twilight_tree_attention(kv, t, t, t, 1, t, n, t, t, ws),
        "window max_new": lambda: B.twilight_window_attention(kv, t, t, t, n, 1, 0, t, t, ws),
        "reserve max_new": lambda: B.twilight_pages_reserve(kv, t, n, t, t, ws),
        "fork new_batch": lambda: B.twilight_pages_fork(kv, t, n, t, t, t, t, t, t, ws),
        "copy n_copy": lambda: B.twilight_pages_copy(kv, t, t, n),
        "compact keep_stride": lambda: B.twilight_tokens_compact(kv, t, t, n, t, t),
        "window": lambda: B.twilight_window_attention(kv, t, t, t, 1, n, 0, t, t, ws),
        "sinks": lambda: B.twilight_window_attention(kv, t, t, t, 1, 1, n, t, t, ws),
    }


@pytest.mark.parametrize("n", [2**31, 2**32 + 4, 2**63 + 1, -2**31 - 1, -2**32 + 5, -2**40])
def test_numbers_beyond_32_bits_are_never_cut_to_them(n, monkeypatch):
    """They are refused; a window and a number of sinks above them are the largest there is, which limits nothing."""
    from paper_2502_02770_amd import binding as B
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: seen.append([a for a in args if isinstance(a, int)]) or 0

    for f in ("_ints", "_rows", "_sums", "_ptr", "_stream_of"):
        monkeypatch.setattr(B, f, lambda t: None)
    monkeypatch.setattr(B, "lib", lambda: Lib())
    for name, call in _calls(B, n).items():
        if n > 0 and name in ("window", "sinks"):
            call()
            assert 2**31 - 1 in seen[-1], name
        else:
            with pytest.raises(AssertionError, match="32 bits"):
                call()
    for call in _calls(B, 7).values():
        call()
        assert 7 in seen[-1]


def test_another_batch_that_does_not_fit_is_refused():
    """Fewer lengths than rows, a table without rows, a pool of another size: the kernels would read past them."""
    import paper_2502_02770_amd as T
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    c, other = object.__new__(T.PagedKV), object.__new__(T.PagedKV)
    c.device, c.num_pool_pages, other.num_pool_pages = torch.device("cpu"), 10, 11
    p = object.__new__(T.PagePool)
    p.cache, p.ref_count, p.status = c, i32(10), i32(1)
    for table, lens in ((i32(4, 5), i32(3)), (i32(4, 5), i32(5)), (i32(20), i32(20)), (i32(2, 2, 5), i32(2))):
        with pytest.raises(AssertionError, match="per row"):
            c.over(table, lens)
    with pytest.raises(AssertionError, match="like"):
        p.over(other)
    assert p.over(c).ref_count is p.ref_count


def test_a_pool_keeps_one_workspace_for_calls_of_all_sizes():
    """Every prompt's length is another max_new, every number of beams another new_batch: what is kept does not grow with them."""
    import paper_2502_02770_amd as T
    from tests.test_new_operators_cpu import _kv
    p = object.__new__(T.PagePool)
    p.cache = object.__new__(T.PagedKV)
    p.cache.kv, p.cache.device = _kv(T, batch=64, max_pages=2048, pool=100000), "cpu"
    p._ws, p._room, rng, given, largest = [], (0, 0), np.random.default_rng(0), [], 0
    for _ in range(2000):
        most, n = (int(rng.integers(1, 32768)), 0) if rng.random() < 0.6 else (0, int(rng.integers(1, 400)))
        ws = p._workspace(most, n)
        need = T.twilight_workspace_bytes(T.TW_WS_PAGES, p.cache.kv, most, n)
        assert ws.numel() >= need > 0
        given.append((ws.data_ptr(), ws.numel()))
        largest = max(largest, need)
    kept = p._ws if isinstance(p._ws, list) else list(p._ws.values())
    assert sum(w.numel() for w in kept) <= 4 * largest
    assert set(given) <= {(w.data_ptr(), w.numel()) for w in kept}            # none that was handed out has gone
    with pytest.raises(AssertionError, match="32 bits"):
        p._workspace(2**32 + 4, 0)
    assert p._workspace(0, 70000).numel() == 0                     # refused by the call; the next one is not short of room
    assert p._workspace(0, 500).numel() >= T.twilight_workspace_bytes(T.TW_WS_PAGES, p.cache.kv, 0, 500)
    assert p._workspace(32767, 399).numel() >= T.twilight_workspace_bytes(T.TW_WS_PAGES, p.cache.kv, 32767, 0)


@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8), (64, 8)])
@pytest.mark.parametrize("new", [1, 4, 16, 128])
def test_workspace_of_new_tokens_follows_the_lists(hq, hkv, new):
    """A list of ceil(pages / 4) tiles has at most half as many parts (528 bytes a row of 32, 64 or 128); and never more than all
    the chip's.  What does not fit a row block is sized for the chip."""
    import paper_2502_02770_amd as T
    from tests.test_new_operators_cpu import _kv
    rows = new * hq // hkv
    block = 32 if rows <= 32 else 64 if rows <= 64 else 128
    size = lambda batch, pages: T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, _kv(T, batch, hq, hkv, pages, 1 << 20), new)
    chip = size(512, 1 << 16)
    for batch, pages in ((1, 1), (1, 256), (2, 300), (3, 9)):
        parts = batch * hkv * -(-(-(-pages // 4)) // 2)
        if rows <= 128:
            assert parts * block * 520 <= size(batch, pages) <= parts * block * 520 + 8 * batch + 512, (batch, pages)
        else:
            assert size(batch, pages) == size(1, 1)
        assert size(batch, pages) <= chip
