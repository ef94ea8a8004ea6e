"""Host-side refusals, workspace sizes and the mask helper of the operators on new tokens and on the cache's pages (no GPU)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from tests.test_kernel_resources_cpu import _fits, kernels  # noqa: F401  (a fixture)


@pytest.fixture(scope="module")
def T():
    import paper_2502_02770_amd as T
    if not os.path.exists(T.binding.LIB_PATH):
        from paper_2502_02770_amd.build import build
        build(verbose=False)
    return T


ONE = ctypes.c_void_p(4096)                                        # never dereferenced: the checks fail first
PLENTY = 1 << 40


def _kv(T, batch=2, hq=32, hkv=8, max_pages=16, pool=64, pools=True, bits=4):
    kv = T.make_kv(batch, hq, hkv, max_pages, pool, None, None, quant_bits=bits)
    kv.page_table = kv.seq_lens = 4096
    if pools:
        kv.k_pool = kv.v_pool = kv.kq_pool = kv.kq_meta = kv.page_minmax = 4096
    return kv


def test_attention_of_new_tokens_refuses(T):
    L, kv = T.binding.lib(), _kv(T)
    ref = ctypes.byref
    tree = lambda kv=kv, q=ONE, max_new=8, mask=ONE, words=1, out=ONE, ws=ONE, n=PLENTY: L.twilight_tree_attention(
        ref(kv), q, None, None, max_new, mask, words, out, None, ws, n, None)
    win = lambda kv=kv, q=ONE, max_new=8, window=64, sinks=4, out=ONE, ws=ONE, n=PLENTY: L.twilight_window_attention(
        ref(kv), q, None, None, max_new, window, sinks, out, None, ws, n, None)
    for f in (tree, win):
        assert f(q=None) == f(out=None) == f(max_new=0) == f(max_new=-1) == f(max_new=(1 << 20) + 1) == -1
        assert f(ws=None) == f(n=16) == -2
        assert f(kv=_kv(T, pools=False)) == -1
        assert f(kv=_kv(T, max_pages=(1 << 24) + 1)) == -1
        bad = _kv(T)
        bad.head_dim = 64
        assert f(kv=bad) == -1
    assert tree(mask=None) == tree(words=0) == tree(max_new=33, words=1) == tree(max_new=1025, words=64) == -1
    assert win(window=0) == win(window=-5) == win(sinks=-1) == -1
    assert win(kv=_kv(T, batch=8000, hq=8, hkv=1), max_new=1 << 20) == -1       # rows beyond 31 bits
    for f in (tree, win):
        for odd in (dict(q=ctypes.c_void_p(4104)), dict(out=ctypes.c_void_p(4100)), dict(ws=ctypes.c_void_p(4097))):
            assert f(**odd) == -1                                  # 16-byte pieces
        odd = _kv(T)
        odd.v_pool = 4104
        assert f(kv=odd) == -1
    no_v = _kv(T)
    no_v.v_pool = None
    assert tree(kv=no_v) == win(kv=no_v) == -1


def test_page_operators_refuse(T):
    L, kv = T.binding.lib(), _kv(T)
    ref = ctypes.byref
    assert L.twilight_pages_reserve(ref(kv), None, 4, ONE, ONE, ONE, PLENTY, None) == -1
    assert L.twilight_pages_reserve(ref(kv), ONE, 0, ONE, ONE, ONE, PLENTY, None) == -1
    assert L.twilight_pages_reserve(ref(kv), ONE, 4, None, ONE, ONE, PLENTY, None) == -1
    assert L.twilight_pages_reserve(ref(kv), ONE, 4, ONE, None, ONE, PLENTY, None) == -1
    assert L.twilight_pages_reserve(ref(kv), ONE, 4, ONE, ONE, None, PLENTY, None) == -2
    assert L.twilight_pages_reserve(ref(kv), ONE, 4, ONE, ONE, ONE, 8, None) == -2
    for k in range(4):
        args = [ONE] * 4
        args[k] = None
        assert L.twilight_pages_free(ref(kv), *args, None) == -1
    fork = lambda parent=ONE, n=3, table=ctypes.c_void_p(8192), lens=ctypes.c_void_p(8192), rc=ONE, src=ONE, dst=ONE, st=ONE, ws=ONE, b=PLENTY: (
        L.twilight_pages_fork(ref(kv), parent, n, table, lens, rc, src, dst, st, ws, b, None))
    for name in ("parent", "table", "lens", "rc", "src", "dst", "st"):
        assert fork(**{name: None}) == -1
    assert fork(n=0) == fork(n=65535) == fork(table=ONE) == fork(lens=ONE) == -1      # in place: the old rows would be read after they change
    assert fork(ws=None) == fork(b=8) == -2
    assert L.twilight_pages_copy(ref(kv), None, ONE, 3, None) == L.twilight_pages_copy(ref(kv), ONE, None, 3, None) == -1
    assert L.twilight_pages_copy(ref(kv), ONE, ONE, -1, None) == -1
    assert L.twilight_pages_copy(ref(kv), ONE, ONE, 0, None) == 0
    for k in (0, 1, 3):
        args = [ONE, ONE, 4, ONE, None]
        args[k] = None
        assert L.twilight_tokens_compact(ref(kv), *args, None) == -1
    assert L.twilight_tokens_compact(ref(kv), ONE, ONE, 0, ONE, None, None) == -1
    assert L.twilight_tokens_compact(ref(_kv(T, pools=False)), ONE, ONE, 4, ONE, None, None) == -1
    big = _kv(T, max_pages=(1 << 24) + 1)
    assert L.twilight_pages_free(ref(big), ONE, ONE, ONE, ONE, None) == -1
    assert L.twilight_tokens_compact(ref(big), ONE, ONE, 4, ONE, None, None) == -1
    odd = _kv(T)
    odd.kq_meta = 4104
    assert L.twilight_pages_copy(ref(odd), ONE, ONE, 3, None) == L.twilight_tokens_compact(ref(odd), ONE, ONE, 4, ONE, None, None) == -1
    no_table = _kv(T)
    no_table.page_table = None
    assert L.twilight_pages_free(ref(no_table), ONE, ONE, ONE, ONE, None) == -1


def test_more_page_requests_than_are_counted_in_32_bits(T):
    L, kv = T.binding.lib(), _kv(T, batch=256, max_pages=1 << 24)
    assert L.twilight_pages_reserve(ctypes.byref(kv), ONE, 2**31 - 1, ONE, ONE, ONE, PLENTY, None) == -1
    kv = _kv(T, batch=128, max_pages=1 << 24)
    assert L.twilight_pages_reserve(ctypes.byref(kv), ONE, 2**31 - 1, ONE, ONE, ONE, PLENTY, None) == -1


def test_workspace_of_a_bound_near_the_largest_int(T):
    """max_new + 15 does not wrap: every page of the pool at most."""
    kv = _kv(T)
    assert 64 * 4 <= T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 2**31 - 1, 0) <= 4096
    assert T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 2**31 - 1, 0) == T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 10**6, 0)


def test_shapes_that_do_not_fit_the_batch_are_refused(T):
    """Before anything reaches the GPU: lists, queries and masks with another number of rows than the cache has."""
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    c = object.__new__(T.PagedKV)
    c.batch, c.Hq, c.kv, c.page_table, c.device = 3, 8, None, i32(3, 5), "cpu"
    p = object.__new__(T.PagePool)
    p.cache = c
    st = object.__new__(T.NewTokens)
    st.cache, st.max_new, st.out = c, 4, torch.zeros(12, 8, 128, dtype=torch.bfloat16)
    q = lambda rows, heads=8: torch.zeros(rows, heads, 128, dtype=torch.bfloat16)
    for call in (lambda: c.copy_pages(i32(4), i32(3)),
                 lambda: c.compact(i32(2, 6), i32(3), i32(3)), lambda: c.compact(i32(3, 6), i32(2), i32(3)), lambda: c.compact(i32(3, 6), i32(3), i32(4)),
                 lambda: c.compact(i32(18), i32(3), i32(3)), lambda: c.compact(i32(3, 6), i32(3), i32(3), i32(3, 4)),
                 lambda: p.reserve(i32(2), 4), lambda: p.free(i32(3), i32(2)), lambda: p.free(i32(2), i32(2)),
                 lambda: st.window(q(3), 64), lambda: st.window(q(12, 4), 64), lambda: st.window(q(12), 64, n_new=i32(2)),
                 lambda: st.tree(q(3), i32(3, 1)), lambda: st.tree(q(12), i32(3, 1)), lambda: st.tree(q(12), i32(12)),
                 lambda: st.tree(q(12), i32(12, 1), n_new=i32(4))):
        with pytest.raises(AssertionError, match="per|batch|like"):
            call()


def test_workspace_sizes_of_the_new_operators(T):
    kv = _kv(T)
    assert T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, kv, 0) == T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, kv, (1 << 20) + 1) == 0
    small, large = (T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, kv, n) for n in (1, 64))
    assert 0 < small < large
    assert T.twilight_workspace_bytes(T.TW_WS_NEW_TOKENS, kv, 1 << 20) == large       # rows beyond a workgroup's do not count
    # a count per row, and every page that can be asked for
    assert T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 33, 0) >= 2 * 4 + 2 * 4 * 4
    assert T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 0, 100) >= 100 * 4 + 64 * 4
    assert T.twilight_workspace_bytes(T.TW_WS_PAGES, kv, 0, 65536) == 0


def test_names_of_the_timed_kernels(T):
    L, names = T.binding.lib(), T.binding.KERNEL_NAMES
    assert [L.twilight_kernel_name(i).decode() for i in range(len(names))] == names and L.twilight_kernel_name(len(names)) == b"?"


def test_the_binding_takes_the_documented_types_only(T):
    for bad in (torch.zeros(4, dtype=torch.int64), torch.zeros(4, 4, dtype=torch.int32).t(), torch.zeros(4, dtype=torch.int32)):
        with pytest.raises(AssertionError):                        # another type, not contiguous, not on the GPU
            T.binding._ints(bad)
    assert T.binding._ints(None) is None


def test_kernels_of_the_new_operators_spill_nothing(kernels):
    """Two workgroups to a compute unit where they have four waves (64 KiB of LDS each), no scratch in any."""
    new = {n: k for n, k in kernels.items() if n.startswith(("new_tokens_", "pages_", "compact_kernel"))}
    assert len(new) == 12 + 6 + 8
    for n, k in new.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
        if n.startswith("new_tokens_kernel"):
            assert _fits(k, 2) and k[".group_segment_fixed_size"] * 2 <= 160 * 1024, (n, k[".vgpr_count"])


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 70])
def test_mask_of_parents(n):
    from paper_2502_02770_amd.cache import tree_mask_of_parents
    rng = np.random.default_rng(n)
    parents = np.stack([[int(rng.integers(-1, j)) if j else -1 for j in range(n)] for _ in range(3)])
    got = tree_mask_of_parents(torch.from_numpy(parents)).numpy()
    assert got.shape == (3, n, -(-n // 32)) and got.dtype == np.int32
    for b in range(3):
        for j in range(n):
            see, k = set(), j
            while k >= 0:
                see.add(k)
                k = int(parents[b, k])
            bits = {w * 32 + i for w in range(got.shape[2]) for i in range(32) if int(got[b, j, w]) >> i & 1}
            assert bits == see
