"""Device buffers for one layer's paged KV cache and for one decode step.

Plumbing only: torch allocates the memory, every computation is a call into
libtwilight.so through `binding`.
"""
import torch

from . import binding as B


class PagedKV:
    """The pools of include/twilight.h's twilight_kv_t, owned as torch tensors."""

    def __init__(self, num_q_heads, num_kv_heads, page_table, seq_lens, num_pool_pages, device="cuda",
                 need_v=True, quant_bits=4, offload_kv=False):
        dev = torch.device(device)
        self.Hq, self.Hkv = int(num_q_heads), int(num_kv_heads)
        self.page_table = page_table.to(dev, torch.int32).contiguous()
        self.seq_lens = seq_lens.to(dev, torch.int32).contiguous()
        self.batch, self.max_pages = self.page_table.shape
        self.num_pool_pages = int(num_pool_pages)
        P, H = self.num_pool_pages, self.Hkv
        # offload_kv: the bf16 K/V pools live in pinned host memory and are read over the host link
        kv_args = dict(dtype=torch.bfloat16, pin_memory=True) if offload_kv else dict(dtype=torch.bfloat16, device=dev)
        self.device = dev
        self.k_pool = torch.zeros(P, H, 16, 128, **kv_args)
        self.v_pool = torch.zeros(P, H, 16, 128, **kv_args) if need_v else None
        self.quant_bits = int(quant_bits)
        self.kq_pool = torch.zeros(P, H, 16, 16 * self.quant_bits, dtype=torch.uint8, device=dev)
        self.kq_meta = torch.zeros(P, H, 16, 4, 2, dtype=torch.float16, device=dev)
        self.page_minmax = torch.zeros(P, H, 2, 128, dtype=torch.bfloat16, device=dev)
        self.kv = B.make_kv(self.batch, self.Hq, self.Hkv, self.max_pages, P, self.page_table, self.seq_lens,
                            self.k_pool, self.v_pool, self.kq_pool, self.kq_meta, self.page_minmax,
                            quant_bits=self.quant_bits)

    def append(self, k_new, v_new, start_pos, n_new, new_offsets, max_new):
        """twilight_kquant_append; does not advance seq_lens."""
        B.twilight_kquant_append(self.kv, k_new, v_new, start_pos, n_new, new_offsets, max_new)

    def fill(self, k, v, seq_offsets):
        """Build the whole cache from logical K/V [total, Hkv, 128] (sequences concatenated)."""
        dev = self.device
        start = torch.zeros(self.batch, dtype=torch.int32, device=dev)
        offs = torch.tensor(seq_offsets[:-1], dtype=torch.int32, device=dev)
        self.append(k, v, start, self.seq_lens, offs, int(self.seq_lens.max().item()))


    def over(self, page_table, seq_lens):
        """A cache of another batch over the same pools (rows of a fork, a larger or smaller batch)."""
        assert page_table.dim() == 2 and seq_lens.numel() == page_table.shape[0], "a length per row of the table"
        c = object.__new__(PagedKV)
        c.__dict__.update(self.__dict__)
        c.page_table = page_table.to(self.device, torch.int32).contiguous()
        c.seq_lens = seq_lens.to(self.device, torch.int32).contiguous()
        c.batch, c.max_pages = c.page_table.shape
        c.kv = B.make_kv(c.batch, c.Hq, c.Hkv, c.max_pages, c.num_pool_pages, c.page_table, c.seq_lens, c.k_pool, c.v_pool,
                         c.kq_pool, c.kq_meta, c.page_minmax, quant_bits=c.quant_bits)
        return c

    def copy_pages(self, src, dst):
        """twilight_pages_copy: whole pages src[i] -> dst[i] of this layer; negative entries are passed over."""
        assert src.shape == dst.shape, "a destination per source"
        B.twilight_pages_copy(self.kv, src, dst, src.numel())

    def compact(self, keep_idx, keep_count, dst_start, dst_table=None):
        """twilight_tokens_compact; does not change seq_lens."""
        assert keep_idx.dim() == 2 and keep_idx.shape[0] == keep_count.numel() == dst_start.numel() == self.batch, "a row per sequence"
        assert dst_table is None or dst_table.shape == self.page_table.shape, "a destination table like the cache's"
        B.twilight_tokens_compact(self.kv, keep_idx, keep_count, keep_idx.shape[1], dst_start, dst_table)


class PagedKV4(PagedKV):
    """A cache held in 4 bits, K and V (twilight_kv4_append and its kind): no bf16 pools; key bounds where with_bounds says so, for the
    page selector, whose quantised K copy this is."""

    def __init__(self, num_q_heads, num_kv_heads, page_table, seq_lens, num_pool_pages, device="cuda", with_bounds=False):
        dev = self.device = torch.device(device)
        self.Hq, self.Hkv, self.num_pool_pages, self.quant_bits = int(num_q_heads), int(num_kv_heads), int(num_pool_pages), 4
        P, H = self.num_pool_pages, self.Hkv
        self.k_pool = self.v_pool = None
        self.kq_pool, self.vq_pool = (torch.zeros(P, H, 16, 64, dtype=torch.uint8, device=dev) for _ in range(2))
        self.kq_meta, self.vq_meta = (torch.zeros(P, H, 16, 4, 2, dtype=torch.float16, device=dev) for _ in range(2))
        self.page_minmax = torch.zeros(P, H, 2, 128, dtype=torch.bfloat16, device=dev) if with_bounds else None
        self._set_batch(page_table, seq_lens)

    def _set_batch(self, page_table, seq_lens):
        assert page_table.dim() == 2 and seq_lens.numel() == page_table.shape[0], "a length per row of the table"
        self.page_table = page_table.to(self.device, torch.int32).contiguous()
        self.seq_lens = seq_lens.to(self.device, torch.int32).contiguous()
        self.batch, self.max_pages = self.page_table.shape
        shape = self.batch, self.Hq, self.Hkv, self.max_pages, self.num_pool_pages, self.page_table, self.seq_lens, None, None
        self.kv = B.make_kv(*shape, self.kq_pool, self.kq_meta, self.page_minmax)
        self._kv_of_v = B.make_kv(*shape, self.vq_pool, self.vq_meta)        # V's codes where those of K are, for what moves rows

    def append(self, k_new, v_new, start_pos, n_new, new_offsets, max_new):
        """twilight_kv4_append; does not advance seq_lens."""
        B.twilight_kv4_append(self.kv, self.vq_pool, self.vq_meta, k_new, v_new, start_pos, n_new, new_offsets, max_new)

    def read(self, start_pos, n_rows, row_offsets, max_rows, k_out, v_out):
        """twilight_kv4_read: rows back as bf16."""
        B.twilight_kv4_read(self.kv, self.vq_pool, self.vq_meta, start_pos, n_rows, row_offsets, max_rows, k_out, v_out)

    def over(self, page_table, seq_lens):
        """A cache of another batch over the same pools (rows of a fork, a larger or smaller batch)."""
        c = object.__new__(PagedKV4)
        c.__dict__.update(self.__dict__)
        c._set_batch(page_table, seq_lens)
        return c

    def copy_pages(self, src, dst):
        """twilight_pages_copy: whole pages src[i] -> dst[i] of this layer; negative entries are passed over."""
        super().copy_pages(src, dst)
        B.twilight_pages_copy(self._kv_of_v, src, dst, src.numel())

    def compact(self, keep_idx, keep_count, dst_start, dst_table=None):
        """twilight_tokens_compact; does not change seq_lens.  Not with key bounds, which the codes do not give back."""
        super().compact(keep_idx, keep_count, dst_start, dst_table)
        B.twilight_tokens_compact(self._kv_of_v, keep_idx, keep_count, keep_idx.shape[1], dst_start, dst_table)


class PagePool:
    """Counts and status word of a pool of pages, shared by the layers whose caches have the same page table.  `cache` is any
    of those layers; the calls change its page_table, or make a new one (fork)."""

    def __init__(self, cache):
        self.cache = cache
        dev = cache.device
        held = cache.page_table[(cache.page_table >= 0) & (cache.page_table < cache.num_pool_pages)].long()
        self.ref_count = torch.bincount(held, minlength=cache.num_pool_pages).to(torch.int32)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self._ws, self._room = [], (0, 0)

    def over(self, cache):
        """The same pool for a cache of another batch (PagedKV.over): counts and status are shared."""
        assert cache.num_pool_pages == self.ref_count.numel(), "a cache over pools like this one's"
        p = object.__new__(PagePool)
        p.cache, p.ref_count, p.status, p._ws = cache, self.ref_count, self.status, []
        p._room = (0, 0)
        return p

    def _workspace(self, max_new, new_batch):
        """One for all calls: its size grows with both arguments.  Outgrown ones are kept, as captured graphs may name them; each is
        at least twice the one before, so that all together are no more than twice the largest."""
        most = tuple(max(x, B._count(y)) for x, y in zip(self._room, (max_new, new_batch)))
        if not self._ws or most != self._room:
            n = B.twilight_workspace_bytes(B.TW_WS_PAGES, self.cache.kv, *most)
            if n == 0:                           # (a size that the call refuses, too)
                return torch.empty(0, dtype=torch.uint8, device=self.cache.device)
            if not self._ws or n > self._ws[-1].numel():
                self._ws.append(torch.empty(max(n, 2 * self._ws[-1].numel() if self._ws else 0), dtype=torch.uint8, device=self.cache.device))
            self._room = most
        return self._ws[-1]

    def reserve(self, n_new, max_new):
        """Pages for the next n_new[b] positions of every sequence (seq_lens not yet advanced)."""
        assert n_new.numel() == self.cache.batch, "a count per sequence"
        B.twilight_pages_reserve(self.cache.kv, n_new, max_new, self.ref_count, self.status, self._workspace(max_new, 0))

    def free(self, first_page, end_page):
        """Logical pages first_page[b] .. end_page[b] - 1 of every row given back."""
        assert first_page.numel() == end_page.numel() == self.cache.batch, "a range per sequence"
        B.twilight_pages_free(self.cache.kv, first_page, end_page, self.ref_count, self.status)

    def free_behind(self, window, num_sinks):
        """The pages given back that neither the sinks nor the window of the next token reaches (twilight_window_attention)."""
        self.free(*pages_behind(self.cache.seq_lens, window, num_sinks))

    def fork(self, parent):
        """-> (new_table, new_lens, copy_src, copy_dst) of the batch whose row i continues row parent[i]; every layer then
        copies the pairs (PagedKV.copy_pages) and goes on over the new table (PagedKV.over, and PagePool.over)."""
        c, n = self.cache, parent.numel()
        i32 = dict(dtype=torch.int32, device=c.device)
        table, lens = torch.empty(n, c.max_pages, **i32), torch.empty(n, **i32)
        src, dst = torch.empty(n, **i32), torch.empty(n, **i32)
        B.twilight_pages_fork(c.kv, parent, n, table, lens, self.ref_count, src, dst, self.status, self._workspace(0, n))
        return table, lens, src, dst


def pages_behind(seq_lens, window, num_sinks):
    """-> (first, end) i32 [batch]: the logical pages of every sequence that lie between the sinks and the window of the next
    token, which stands at position seq_lens[b].  Windows and sinks of any size, as NewTokens.window takes them."""
    assert window >= 1 and num_sinks >= 0, "a window of one token at least, and no fewer than no sinks"
    window, num_sinks = min(int(window), 2**31 - 1), min(int(num_sinks), 2**31 - 1)
    # (differences of two numbers that are not negative stay in 32 bits)
    behind = torch.clamp(torch.clamp(seq_lens, min=0) - (window - 1), min=0)
    return torch.full_like(seq_lens, -(-num_sinks // 16)), behind // 16


class NewTokens:
    """Pre-allocated outputs and workspace of attention of up to max_new new tokens per sequence (rows b * max_new + i)."""

    def __init__(self, cache, max_new, with_lse=True):
        c = self.cache = cache
        self.max_new = int(max_new)
        rows = c.batch * self.max_new
        self.out = torch.zeros(rows, c.Hq, 128, dtype=torch.bfloat16, device=c.device)
        self.lse = torch.zeros(rows, c.Hq, dtype=torch.float32, device=c.device) if with_lse else None
        self.ws = torch.empty(B.twilight_workspace_bytes(B.TW_WS_KV4 if isinstance(c, PagedKV4) else B.TW_WS_NEW_TOKENS, c.kv, self.max_new),
                              dtype=torch.uint8, device=c.device)

    def _check(self, q, n_new):
        assert q.shape == self.out.shape, "q [batch * max_new, heads, 128]"
        assert n_new is None or n_new.numel() == self.cache.batch, "a count per sequence"

    def tree(self, q, tree_mask, n_new=None):
        """A drafted tree per sequence; tree_mask i32 [rows, words] (tree_mask_of_parents)."""
        self._check(q, n_new)
        assert not isinstance(self.cache, PagedKV4), "trees are read from bf16 pools"
        assert tree_mask.dim() == 2 and tree_mask.shape[0] == q.shape[0], "a mask row per row of q"
        B.twilight_tree_attention(self.cache.kv, q, n_new, None, self.max_new, tree_mask, tree_mask.shape[1], self.out, self.lse, self.ws)
        return self.out

    def window(self, q, window, num_sinks=0, n_new=None):
        """Consecutive tokens under a sliding window with sinks."""
        self._check(q, n_new)
        c = self.cache
        if isinstance(c, PagedKV4):
            B.twilight_kv4_attention(c.kv, c.vq_pool, c.vq_meta, q, n_new, None, self.max_new, window, num_sinks, self.out, self.lse, self.ws)
        else:
            B.twilight_window_attention(c.kv, q, n_new, None, self.max_new, window, num_sinks, self.out, self.lse, self.ws)
        return self.out


class TokenMass:
    """The attention that every token of a layer's cache (PagedKV or PagedKV4) has got, and what it is worth keeping by it."""

    def __init__(self, cache):
        c = self.cache = cache
        self.mass, self._spare = (torch.zeros(c.batch, c.max_pages * 16, dtype=torch.float32, device=c.device) for _ in range(2))
        self.keep_idx = torch.zeros(c.batch, c.max_pages * 16, dtype=torch.int32, device=c.device)
        self.keep_count, self._start = (torch.zeros(c.batch, dtype=torch.int32, device=c.device) for _ in range(2))
        self.ws = torch.empty(B.twilight_workspace_bytes(B.TW_WS_KEEP, c.kv), dtype=torch.uint8, device=c.device)

    def add(self, q, lse, max_new, window=2**31 - 1, num_sinks=0, n_new=None, new_offsets=None, decay=1.0):
        """What the newest tokens' attention gave (twilight_attention_mass); q, lse and the rest as of the attention call."""
        assert n_new is None or n_new.numel() == self.cache.batch, "a count per sequence"
        assert lse.numel() * 128 == q.numel() and (new_offsets is not None or q.shape[0] >= self.cache.batch * max_new), "a row per new token"
        B.twilight_attention_mass(self.cache.kv, q, lse, n_new, new_offsets, max_new, window, num_sinks, decay, self.mass, self.mass)

    def keep(self, budget, num_sinks=0, num_recent=0):
        """-> (keep_idx [batch, max_pages * 16], keep_count): the tokens worth most (twilight_keep_tokens)."""
        self._spare.zero_()                        # (tokens that come behind the kept ones begin with nothing)
        B.twilight_keep_tokens(self.cache.kv, self.mass, budget, num_sinks, num_recent, self.keep_idx, self.keep_count, self.keep_idx.shape[1],
                               self._spare, self.ws)
        return self.keep_idx, self.keep_count

    def evict(self, budget, num_sinks=0, num_recent=0, others=()):
        """Every sequence cut down to its budget: the tokens worth keeping moved together in place, seq_lens set to their number, and
        their mass kept for the steps to come.  The pages behind are the caller's to give back (PagePool.free), and no page may be
        shared with another sequence.  Layers whose caches have one seq_lens tensor between them (as those of one PagedKV.over) are cut
        down by one call, each by its own mass: `others` are the TokenMass of the rest of them.  In a call of its own, a later layer would
        find the lengths set already, and choose from the first of its tokens alone.  -> keep_count"""
        layers = (self, *others)
        assert all(m.cache.batch == self.cache.batch for m in layers), "layers of one batch"
        for m in layers:
            m.keep(budget, num_sinks, num_recent)
            m.cache.compact(m.keep_idx, m.keep_count, m._start)
        for m in layers:
            m.cache.seq_lens.copy_(m.keep_count)
            m.mass.copy_(m._spare)                 # (not exchanged: a captured graph names them)
        return self.keep_count


def tree_mask_of_parents(parents):
    """Mask words [..., ceil(n / 32)] (i32) of drafted trees from their parents [..., n] (before their children; -1, or whatever
    else is no token before the child: the last cached token): every token sees its ancestors and itself.
    In steps that double the ancestors found: 8 drafts of 128 tokens 0.29 ms, 6.3 ms a token at a time."""
    n = parents.shape[-1]
    j = torch.arange(n, device=parents.device)
    # row n is the cache's: no bits, and its own parent.  With every step a row takes over what its 2^k nearest ancestors see.
    up = torch.where((parents >= 0) & (parents < j), parents.long(), torch.full_like(j, n))
    up = torch.cat([up, torch.full_like(up[..., :1], n)], -1) if n else up
    bit = torch.where(j % 32 == 31, torch.full_like(j, -1 << 31), 1 << j % 32).to(torch.int32)
    words = torch.where(j[:, None] // 32 == torch.arange(-(-n // 32), device=j.device), bit[:, None], torch.zeros_like(bit[:, None]))
    words = torch.cat([words, torch.zeros_like(words[:1])]).expand(*parents.shape[:-1], -1, -1)
    for _ in range((n - 1).bit_length() if n else 0):
        words = words | words.gather(-2, up[..., None].expand(words.shape))
        up = up.gather(-1, up)
    return words[..., :n, :].contiguous()


class DecodeStep:
    """Pre-allocated outputs and workspaces of one decode step; runs
    select -> prune -> attend through the C ABI."""

    def __init__(self, cache, max_sel=None, union_stride=None, with_kept_idx=False, with_lse=True):
        c, dev = cache, cache.device
        self.cache = c
        self.full = max_sel is None
        self.max_sel = 0 if self.full else int(max_sel)
        cand = (c.max_pages if self.full else self.max_sel) * 16
        G = c.Hq // c.Hkv
        self.union_stride = int(union_stride) if union_stride else min(G * cand, c.max_pages * 16)
        i32 = dict(dtype=torch.int32, device=dev)
        if not self.full:
            self.sel_pages = torch.zeros(c.batch, c.Hq, self.max_sel, **i32)
            self.sel_count = torch.zeros(c.batch, c.Hq, **i32)
            # one allocation for the selector's and the pruner's workspaces, laid out as twilight_select_prune wants
            # them; the separate calls get its two parts
            nsel = B.twilight_workspace_bytes(B.TW_WS_SELECT, c.kv, self.max_sel)
            self._ws_select_prune = torch.empty(B.twilight_workspace_bytes(B.TW_WS_SELECT_PRUNE, c.kv, self.max_sel),
                                                dtype=torch.uint8, device=dev)
            self.ws_select = self._ws_select_prune[:nsel]
            self.ws_prune = self._ws_select_prune[nsel:]
        else:
            self.sel_pages = self.sel_count = None
        self.kept_count = torch.zeros(c.batch, c.Hq, **i32)
        self.kept_stride = cand if with_kept_idx else 0
        self.kept_idx = torch.zeros(c.batch, c.Hq, cand, **i32) if with_kept_idx else None
        self.union_count = torch.zeros(c.batch * c.Hkv, **i32)
        self.union_idx = torch.zeros(c.batch * c.Hkv, self.union_stride, **i32)
        self.status = torch.zeros(1, **i32)
        if self.full:
            self.ws_prune = torch.empty(B.twilight_workspace_bytes(B.TW_WS_PRUNE, c.kv, self.max_sel), dtype=torch.uint8, device=dev)
        self.ws_decode = torch.empty(B.twilight_workspace_bytes(B.TW_WS_DECODE, c.kv, 0, self.union_stride), dtype=torch.uint8, device=dev)
        self.out = torch.zeros(c.batch, c.Hq, 128, dtype=torch.bfloat16, device=dev)
        self.lse = torch.zeros(c.batch, c.Hq, dtype=torch.float32, device=dev) if with_lse else None
        self._ws_dense = None
        self._ws_per_head = None

    def select(self, q, budget):
        B.twilight_select_pages(self.cache.kv, q, budget, self.sel_pages, self.sel_count, self.max_sel, self.ws_select)

    def append_select(self, k_new, v_new, new_pos, q, budget):
        """One new token per sequence appended and the pages selected in one launch."""
        B.twilight_append_select(self.cache.kv, k_new, v_new, new_pos, q, budget, self.sel_pages, self.sel_count,
                                 self.max_sel, self.ws_select)

    def select_prune(self, k_new, v_new, new_pos, q, budget, p):
        """Selector (with the step's new token appended when k_new is given) and pruner in two launches."""
        B.twilight_select_prune(self.cache.kv, k_new, v_new, new_pos, q, budget, p, self.sel_pages, self.sel_count,
                                self.max_sel, self.kept_count, self.kept_idx, self.kept_stride, self.union_count,
                                self.union_idx, self.union_stride, self.status, self._ws_select_prune)

    def prune(self, q, p):
        B.twilight_topp_prune(self.cache.kv, q, self.sel_pages, self.sel_count, self.max_sel, p, self.kept_count,
                              self.kept_idx, self.kept_stride, self.union_count, self.union_idx,
                              self.union_stride, self.status, self.ws_prune)

    def attend(self, q):
        B.twilight_sparse_decode(self.cache.kv, q, self.union_count, self.union_idx, self.union_stride, self.out,
                                 self.lse, self.ws_decode)

    def attend_per_head(self, q):
        """Every query head over its own kept set (needs with_kept_idx=True) instead of the group's union."""
        assert self.kept_idx is not None, "DecodeStep(with_kept_idx=True) keeps the per-head lists"
        if self._ws_per_head is None:
            self._ws_per_head = torch.empty(
                B.twilight_workspace_bytes(B.TW_WS_DECODE_PER_HEAD, self.cache.kv, 0, self.kept_stride),
                dtype=torch.uint8, device=self.out.device)
        B.twilight_sparse_decode_per_head(self.cache.kv, q, self.kept_count, self.kept_idx, self.kept_stride,
                                          self.out, self.lse, self._ws_per_head)

    def run(self, q, budget, p, separate=False):
        """Selector, pruner, attention.  With a page selector the first two are one call (twilight_select_prune);
        separate=True takes twilight_select_pages and twilight_topp_prune instead (same results bit for bit)."""
        if self.full:
            self.prune(q, p)
        elif separate:
            self.select(q, budget)
            self.prune(q, p)
        else:
            self.select_prune(None, None, None, q, budget, p)
        self.attend(q)
        return self.out

    def dense(self, q, out=None, lse=None):
        """Dense decode attention over all tokens through the same kernel (baseline)."""
        c = self.cache
        if self._ws_dense is None:
            self._ws_dense = torch.empty(B.twilight_workspace_bytes(B.TW_WS_DECODE, c.kv, 0, 0), dtype=torch.uint8,
                                         device=c.device)
        out = self.out if out is None else out
        B.twilight_sparse_decode(c.kv, q, None, None, 0, out, lse, self._ws_dense)
        return out
