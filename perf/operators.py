"""Cases for timing the operators on new tokens and on the cache's pages, and those operators in plain torch.

  tree      attention of a drafted tree of tokens over a sequence's paged cache
  window    attention of the newest tokens of a sequence (one, a chunk, a whole prompt) with a sliding window and a few
            first tokens that stay visible
  accept    a drafted branch's pages copied for a sequence of its own, and the accepted tokens moved up in them
  evict     the kept tokens of every sequence packed into other pages
  fork      a batch's sequences rearranged into another batch by parent rows (beams, parallel samples), pages shared,
            the partly filled ones copied
  turn      a serving step's pages: those of finished and passed tokens given back, those of new tokens handed out

The cache is the paged one of this package: pages of 16 tokens, head_dim 128, bf16 K and V, a quantised copy of K with
fp16 (scale, zero) per 32 dims, and per page the element-wise bounds of K.
"""
import math
import random

import numpy as np
import torch

own = False

D, PAGE = 128, 16
SCALE = 1.0 / math.sqrt(D)


# ---------------------------------------------------------------------------------------------------------------- cases
def _attn(name, op, batch, tokens, new, q_heads=32, kv_heads=8, ragged=False, window=0, sinks=0, lens_seed=0):
    c = dict(op=op, batch=batch, tokens=tokens, new=new, q_heads=q_heads, kv_heads=kv_heads, ragged=ragged, window=window,
             sinks=sinks, lens_seed=lens_seed)
    return c if name is None else dict(c, name=name)


def _pages(name, op, batch, tokens, new=0, kv_heads=8, keep=0.5, spare=0.25, bits=4, lens_seed=0):
    c = dict(op=op, batch=batch, tokens=tokens, new=new, q_heads=kv_heads, kv_heads=kv_heads, keep=keep, spare=spare, bits=bits,
             lens_seed=lens_seed)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a single chat with a short draft: launch and dependency latency
        _attn("tree_1x4k_8", "tree", 1, 4096, 8),
        # the ordinary serving batch, verified with trees of 32
        _attn("tree_8x32k_32", "tree", 8, 32768, 32),
        # requests of odd lengths with trees of up to 61 tokens on a wide model, some with no draft at all
        _attn("tree_ragged_61_g8", "tree", 13, 16001, 61, q_heads=64, ragged=True, lens_seed=7),
        # a multi-head model (every query head its own KV head), trees of 16
        _attn("tree_mha_4x8k_16", "tree", 4, 8192, 16, kv_heads=32),
        # one chat's next token in a layer with a window
        _attn("window_1x4k", "window", 1, 4096, 1, window=1024, sinks=4),
        # mixed traffic, one token each
        _attn("window_ragged64", "window", 64, 32768, 1, ragged=True, window=4096, sinks=16, lens_seed=5),
        # chunked prefill behind long contexts of odd lengths, wide model
        _attn("window_chunk_odd_g8", "window", 3, 9001, 1499, q_heads=64, window=2047, sinks=5),
        # whole prompts
        _attn("window_prompt_2x8k", "window", 2, 8192, 8192, window=4096, sinks=4),
        # the end of a speculative step in one layer
        _pages("accept_8x64", "accept", 8, 1000, 64, keep=0.3),
        # half of a long context given up
        _pages("evict_4x16k", "evict", 4, 16384, keep=0.5),
        # beams: parents drawn again, pages shared, partial pages copied
        _pages("fork_48", "fork", 48, 4000, spare=0.2, lens_seed=2),
        # pages of a serving step over a large pool
        _pages("turn_64x32k", "turn", 64, 32768, 300, lens_seed=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["tree"] * 3 + ["window"] * 4 + ["accept", "evict", "fork", "turn"])
    seed = rng.randrange(1 << 30)
    if op in ("tree", "window"):
        q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (64, 8), (32, 32), (16, 8)])
        if op == "tree":
            new = _log_int(rng, 1, 128)
            batch = _log_int(rng, 1, 32)
            # K/V rows and scores (new tokens x tokens x query heads) of the largest listed cases
            top = min((1 << 21) // kv_heads, (1 << 28) // (new * q_heads)) // batch
            return _attn(None, op, batch, _log_int(rng, 300, max(400, min(65536, top))), new, q_heads, kv_heads,
                         ragged=rng.random() < 0.5, lens_seed=seed)
        kind = rng.choice(["one", "chunk", "prompt"])
        sinks = rng.choice([0, 1, 4, 16, 64])
        if kind == "one":
            batch = _log_int(rng, 1, 64)
            tokens = _log_int(rng, 300, max(400, min(65536, (1 << 23) // kv_heads // batch)))
            new = 1
        else:
            batch = _log_int(rng, 1, 8)
            tokens = _log_int(rng, 300, 9000)
            new = min(tokens, max(2, (1 << 31) // (tokens * q_heads * batch)), tokens if kind == "prompt" else _log_int(rng, 2, 2048))
        return _attn(None, op, batch, tokens, new, q_heads, kv_heads, ragged=rng.random() < 0.5, window=_log_int(rng, 16, 8192),
                     sinks=sinks, lens_seed=seed)
    kv_heads = rng.choice([8, 8, 32, 4])
    bits = rng.choice([4, 4, 4, 8, 2])
    if op == "accept":
        return _pages(None, op, _log_int(rng, 1, 32), _log_int(rng, 20, 1000), _log_int(rng, 1, 128), kv_heads,
                      keep=rng.choice([0.05, 0.3, 0.9]), bits=bits, lens_seed=seed)
    if op == "evict":
        batch = _log_int(rng, 1, 16)
        return _pages(None, op, batch, _log_int(rng, 100, (1 << 19) // kv_heads // batch), 0, kv_heads, keep=rng.choice([0.1, 0.5, 0.8]),
                      bits=bits, lens_seed=seed)
    if op == "fork":
        return _pages(None, op, _log_int(rng, 2, 64), _log_int(rng, 40, 4000 * 8 // max(8, kv_heads)), 0, kv_heads,
                      spare=rng.choice([0.05, 0.2, 0.5]), bits=bits, lens_seed=seed)
    return _pages(None, op, _log_int(rng, 1, 64), _log_int(rng, 100, 32768), _log_int(rng, 1, 300), 8, lens_seed=seed)


def _lens(case):
    """Tokens of each sequence, and how many of them are new."""
    n, b, new = case["tokens"], case["batch"], case["new"]
    if not case.get("ragged"):
        return [n] * b, [min(new, n)] * b
    r = random.Random(case["lens_seed"])
    lens = [_log_int(r, max(1, n // 32), n) for _ in range(b)]
    many = [min(x, r.choice([new, new, r.randint(1, new), 1, 0 if new > 1 else 1])) for x in lens]
    many[0] = min(new, lens[0])
    return lens, many


def _odd_lens(case, lo=None):
    """Lengths of the page cases: odd ones from half the case's tokens on."""
    r = random.Random(case["lens_seed"])
    return [r.randint(max(1, case["tokens"] // 2 if lo is None else lo), case["tokens"]) for _ in range(case["batch"])]


def _page_bytes(case):
    return case["kv_heads"] * PAGE * (2 * D * 2 + 16 * case["bits"] + 16) + case["kv_heads"] * 2 * D * 2


def _visible(case, n, new):
    """(positions that any of the new tokens sees, pairs of a new token and a position) of a sequence."""
    if case["op"] == "tree":
        return (n if new else 0), new * (n - new) + new
    p = np.arange(n - new, n, dtype=np.int64)
    sinks = np.minimum(case["sinks"], np.maximum(0, p + 1 - case["window"]))
    first = max(0, n - new - case["window"] + 1) if new else 0
    return (n - first + min(case["sinks"], first) if new else 0), int((np.minimum(case["window"], p + 1) + sinks).sum())


def work(case):
    op, hq, hkv = case["op"], case["q_heads"], case["kv_heads"]
    if op in ("tree", "window"):
        lens, many = _lens(case)
        seen = [_visible(case, n, m) for n, m in zip(lens, many)]
        rows = sum(many)
        small = rows * hq * (2 * D * 2 + 4) + (rows * 4 * -(-max(case["new"], 1) // 32) if op == "tree" else 0) + sum(-(-n // PAGE) * 4 for n in lens)
        return {"bytes": sum(s[0] for s in seen) * hkv * D * 4 + small, "flops": 4.0 * D * hq * sum(s[1] for s in seen)}
    token = hkv * (2 * D * 2 + 16 * case["bits"] + 16)
    lens = _odd_lens(case)
    if op == "accept":
        kept = case["batch"] * max(1, int(case["keep"] * case["new"]))
        pages = sum((n + case["new"] - 1) // PAGE - n // PAGE + 1 for n in lens)
        return {"bytes": 2.0 * pages * _page_bytes(case) + 2.0 * kept * token, "flops": 0.0}
    if op == "evict":
        kept = sum(max(1, int(case["keep"] * n)) for n in lens)
        return {"bytes": 2.0 * kept * token + kept / PAGE * hkv * 2 * D * 2 + kept * 4, "flops": 0.0}
    if op == "fork":
        table = case["batch"] * -(-case["tokens"] // PAGE) * 4
        return {"bytes": 2.0 * table + 2 * 4 * _pool_pages(case) + 2.0 * case["batch"] // 3 * _page_bytes(case), "flops": 0.0}
    return {"bytes": 2.0 * 4 * case["batch"] * _turn_pages(case) + 2.0 * 4 * _pool_pages(case), "flops": 0.0}


def _turn_pages(case):
    return -(-(case["tokens"] + case["new"]) // PAGE)


def _pool_pages(case):
    """Pages of the pool of a fork or a turn."""
    lens = _odd_lens(case)
    held = sum(-(-n // PAGE) for n in lens)
    return held + case["batch"] + int(case["spare"] * held) + case["batch"] * (-(-case["new"] // PAGE) + 1)


# --------------------------------------------------------------------------------------------------------------- inputs
def _i32(x, dev="cuda"):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(dev)


def _pools(P, hkv, bits, g, with_codes):
    dev = "cuda"
    s = dict(k=torch.randn(P, hkv, PAGE, D, device=dev, dtype=torch.bfloat16, generator=g),
             v=torch.randn(P, hkv, PAGE, D, device=dev, dtype=torch.bfloat16, generator=g))
    if with_codes:
        s["codes"] = torch.randint(0, 256, (P, hkv, PAGE, 16 * bits), device=dev, dtype=torch.uint8, generator=g)
        s["meta"] = torch.randn(P, hkv, PAGE, 4, 2, device=dev, dtype=torch.float16, generator=g)
        s["bounds"] = torch.stack([s["k"].amin(2), s["k"].amax(2)], 2).contiguous()
    return s


def _table(lens, max_pages, rng, extra=0):
    """Pages of all sequences in shuffled order; [batch, max_pages], -1 beyond a sequence's pages. -> (table, pages in use)"""
    held = [-(-n // PAGE) for n in lens]
    ids = rng.permutation(sum(held) + extra)
    table = np.full((len(lens), max_pages), -1, dtype=np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    return table, ids, at


def _trees(many, new, rng):
    """Ancestors-and-self masks of random trees, i32 words [rows, ceil(new / 32)]."""
    words = -(-new // 32)
    rows = []
    for m in many:
        see = np.zeros((m, words * 32), dtype=np.uint8)
        for j in range(m):
            up = int(rng.integers(max(-1, j - 8), j)) if j else -1
            if up >= 0:
                see[j] = see[up]
            see[j, j] = 1
        rows.append(np.packbits(see, axis=1, bitorder="little").view("<i4"))
    return np.concatenate(rows).reshape(-1, words)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    op, hq, hkv = case["op"], case["q_heads"], case["kv_heads"]
    s = dict(op=op, Hq=hq, Hkv=hkv, batch=case["batch"], bits=case.get("bits", 4))
    if op in ("tree", "window"):
        lens, many = _lens(case)
        max_pages = -(-max(lens) // PAGE)
        table, _, used = _table(lens, max_pages, rng)
        s.update(_pools(used, hkv, 4, g, False), table=_i32(table), lens=_i32(lens), n_new=_i32(many),
                 offsets=_i32(np.cumsum([0] + many[:-1])), max_new=case["new"], window=case["window"], sinks=case["sinks"],
                 # queries of different sharpness, from even to peaked attention
                 q=(torch.randn(sum(many), hq, D, device="cuda", generator=g)
                    * (0.5 + 2.5 * torch.rand(1, hq, 1, device="cuda", generator=g))).to(torch.bfloat16))
        if op == "tree":
            s["mask"] = _i32(_trees(many, case["new"], rng))
        return s
    lens = _odd_lens(case)
    if op == "accept":
        # context of lens[b] tokens, `new` drafted ones behind it; the drafted tail's pages are to be copied to the sequence's own
        new, kept = case["new"], max(1, int(case["keep"] * case["new"]))
        full = [n + new for n in lens]
        tails = [(n // PAGE, -(-(n + new) // PAGE)) for n in lens]
        max_pages = -(-max(full) // PAGE)
        table, ids, at = _table(full, max_pages, rng, extra=sum(b - a for a, b in tails))
        src, dst = [], []
        for b, (lo, hi) in enumerate(tails):
            src += table[b, lo:hi].tolist()
            dst += ids[at:at + hi - lo].tolist()
            table[b, lo:hi] = ids[at:at + hi - lo]
            at += hi - lo
        keep = np.stack([n + np.sort(rng.permutation(new)[:kept]) for n in lens])
        s.update(_pools(len(ids), hkv, case["bits"], g, True), table=_i32(table), lens=_i32(full), src=_i32(src), dst=_i32(dst),
                 keep=_i32(keep), count=_i32([kept] * len(lens)), start=_i32(lens))
        return s
    if op == "evict":
        kept = [max(1, int(case["keep"] * n)) for n in lens]
        max_pages = -(-max(lens) // PAGE)
        table, ids, at = _table(lens, max_pages, rng, extra=sum(-(-k // PAGE) for k in kept))
        to = np.full_like(table, -1)
        keep = np.full((len(lens), max(kept)), -1, dtype=np.int32)
        for b, k in enumerate(kept):
            to[b, :-(-k // PAGE)] = ids[at:at - (-k // PAGE)]
            at += -(-k // PAGE)
            keep[b, :k] = np.sort(rng.permutation(lens[b])[:k])
        s.update(_pools(len(ids), hkv, case["bits"], g, True), table=_i32(table), to=_i32(to), lens=_i32(lens), keep=_i32(keep),
                 count=_i32(kept), start=_i32([0] * len(lens)))
        return s
    pool = _pool_pages(case)
    if op == "fork":
        max_pages = -(-case["tokens"] // PAGE)
        table, ids, at = _table(lens, max_pages, rng, extra=pool - sum(-(-n // PAGE) for n in lens))
        b = case["batch"]
        parent = np.where(rng.random(b) < 0.6, np.arange(b), rng.integers(0, b, b))
        parent[rng.random(b) < 0.05] = -1
        s.update(_pools(pool, hkv, case["bits"], g, True), table=_i32(table), lens=_i32(lens), parent=_i32(parent))
    else:
        max_pages = _turn_pages(case)
        table, ids, at = _table(lens, max_pages, rng, extra=pool - sum(-(-n // PAGE) for n in lens))
        first = rng.integers(0, 5, len(lens))                       # some sequences end, others move their window on
        end = np.where(rng.random(len(lens)) < 0.15, max_pages, first + rng.integers(0, 6, len(lens)))
        first = np.where(end == max_pages, 0, first)
        now = np.where(end == max_pages, 0, lens)
        many = np.where(end == max_pages, rng.integers(1, case["new"] + 1, len(lens)), rng.integers(0, 2, len(lens)))
        s.update(table=_i32(table), lens=_i32(now), first=_i32(first), end=_i32(end), n_new=_i32(many), max_new=case["new"])
    ref = np.zeros(pool, dtype=np.int32)
    np.add.at(ref, table[table >= 0], 1)
    s.update(ref=_i32(ref), pool=pool)
    return s


# ------------------------------------------------------------------------------------------------------- the operators
def run(state):
    if own:
        return _run_own(state)
    return dict(tree=_plain_attention, window=_plain_attention, accept=_plain_accept, evict=_plain_evict, fork=_plain_fork,
                turn=_plain_turn)[state["op"]](state)


def _plain_attention(s):
    B, Hq, Hkv, T = s["batch"], s["Hq"], s["Hkv"], s["max_new"]
    G, L, dev = Hq // Hkv, s["table"].shape[1] * PAGE, s["q"].device
    pages = s["table"].long().clamp(0, s["k"].shape[0] - 1)
    k = s["k"][pages].transpose(2, 3).reshape(B, L, Hkv, D).transpose(1, 2).float().contiguous()        # [B, Hkv, L, D]
    v = s["v"][pages].transpose(2, 3).reshape(B, L, Hkv, D).transpose(1, 2).float().contiguous()
    lens, many, offs = s["lens"].long(), s["n_new"].long(), s["offsets"].long()
    i, t = torch.arange(T, device=dev), torch.arange(L, device=dev)
    rows = (offs[:, None] + i).clamp(max=s["q"].shape[0] - 1)                                             # [B, T]
    ctx = (lens - many)[:, None, None]
    if s["op"] == "tree":
        j = t - ctx                                                                                       # [B, 1, L]
        at = j.clamp(0, s["mask"].shape[1] * 32 - 1).expand(B, T, L)
        word = torch.gather(s["mask"].long()[rows], 2, at // 32)
        see = (j < 0) | (((word >> (at % 32)) & 1) == 1) & (j < many[:, None, None])
    else:
        p = ctx + i[:, None]                                                                              # [B, T, 1]
        see = (t <= p) & ((p - t < s["window"]) | (t < s["sinks"]))
    see = see & (t < lens[:, None, None])
    q = s["q"][rows].float().view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D)
    x = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, G, T, L).mul_(SCALE)
    x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (m + total.log()).squeeze(-1)                                                                   # log 0 = -inf
    o = torch.matmul(x.view(B, Hkv, G * T, L), v).view(B, Hkv, G, T, D) / torch.where(total == 0, torch.ones_like(total), total)
    # back to the rows of q
    r = torch.arange(s["q"].shape[0], device=dev)
    b = torch.searchsorted((offs + many).contiguous(), r, right=True).clamp(max=B - 1)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)[b, r - offs[b]]
    lse = lse.permute(0, 3, 1, 2).reshape(B, T, Hq)[b, r - offs[b]]
    return {"out": o.to(torch.bfloat16), "lse": lse}


def _all_pools(s):
    return [s["k"], s["v"], s["codes"], s["meta"], s["bounds"]]


def _plain_copy(s, src, dst):
    """Pages src -> dst in every pool; pairs with a negative page (src) do nothing: they stand for a page copied to itself."""
    dst = torch.where(src < 0, torch.zeros_like(dst), dst).long()
    src = torch.where(src < 0, torch.zeros_like(src), src).long()
    first = torch.argmax((src != dst).int())                         # a pair that does nothing repeats one that does something
    idle = src == dst
    src, dst = torch.where(idle, src[first], src), torch.where(idle, dst[first], dst)
    s["k"][dst], s["v"][dst], s["codes"][dst] = s["k"][src], s["v"][src], s["codes"][src]
    s["meta"][dst], s["bounds"][dst] = s["meta"][src], s["bounds"][src]


def _plain_compact(s, to):
    keep, count, start = s["keep"].long(), s["count"].long(), s["start"].long()
    B, N = keep.shape
    i = torch.arange(N, device=keep.device)
    idle = i >= count[:, None]                                       # repeats the first kept token's move
    frm = torch.where(idle, keep[:, :1], keep)
    onto = start[:, None] + torch.where(idle, torch.zeros_like(keep), i)
    sp, ss = torch.gather(s["table"].long(), 1, frm // PAGE), frm % PAGE
    dp, ds = torch.gather(to.long(), 1, onto // PAGE), onto % PAGE
    moved = s["k"][sp, :, ss], s["v"][sp, :, ss], s["codes"][sp, :, ss], s["meta"][sp, :, ss]
    s["k"][dp, :, ds], s["v"][dp, :, ds], s["codes"][dp, :, ds], s["meta"][dp, :, ds] = moved
    # bounds of the pages that hold the moved tokens, over the tokens up to the new end
    last = (start + count - 1)[:, None]
    lp = torch.minimum(start[:, None] // PAGE + torch.arange(-(-N // PAGE) + 1, device=keep.device), last // PAGE)
    page = torch.gather(to.long(), 1, lp)
    held = (lp[..., None] * PAGE + torch.arange(PAGE, device=keep.device) <= last[..., None])[:, :, None, :, None]
    rows = s["k"][page].float()
    lo = torch.where(held, rows, torch.full_like(rows, math.inf)).amin(3)
    hi = torch.where(held, rows, torch.full_like(rows, -math.inf)).amax(3)
    s["bounds"][page] = torch.stack([lo, hi], 3).to(torch.bfloat16)


def _plain_accept(s):
    _plain_copy(s, s["src"], s["dst"])
    _plain_compact(s, s["table"])
    return _all_pools(s)


def _plain_evict(s):
    _plain_compact(s, s["to"])
    return _all_pools(s)


def _lowest_free(ref, wants):
    """wants: truth values in the order in which pages are asked for. -> their pages (-1 where none is wanted or left), the new counts"""
    want = wants.reshape(-1)
    rank = torch.cumsum(want.long(), 0) - 1
    free = ref == 0
    nth = torch.cumsum(free.long(), 0) - 1
    P = ref.numel()
    listing = torch.full((P + 1,), -1, dtype=torch.long, device=ref.device)
    listing.scatter_(0, torch.where(free, nth, torch.full_like(nth, P)), torch.arange(P, device=ref.device))
    listing[P] = -1
    got = torch.where(want, listing[rank.clamp(0, P)], torch.full_like(rank, -1))
    return got.view(wants.shape), torch.where(free & (nth < want.sum()), torch.ones_like(ref), ref)


def _plain_fork(s):
    table, lens, parent = s["table"].long(), s["lens"].long(), s["parent"].long()
    B, MP = table.shape
    P, dev = s["pool"], table.device
    from_ = parent.clamp(min=0)
    lp = torch.arange(MP, device=dev)
    children = torch.zeros(B + 1, dtype=torch.long, device=dev).scatter_add_(0, torch.where(parent < 0, torch.full_like(parent, B), parent), torch.ones_like(parent))[:B]
    earlier = (parent[:, None] == parent[None, :]) & (torch.arange(B, device=dev)[None, :] < torch.arange(B, device=dev)[:, None])
    first = (parent >= 0) & ~earlier.any(1)
    rows = table[from_]
    shared = lp < (lens[from_] // PAGE)[:, None]
    new = torch.where((parent >= 0)[:, None] & (shared | first[:, None]), rows, torch.full_like(rows, -1))
    # references: whole pages by the number of children, the others by whether there is one
    whole = lp < (lens // PAGE)[:, None]
    delta = torch.where(whole, (children - 1)[:, None], -(children == 0).long()[:, None])
    flat = torch.zeros(P + 1, dtype=torch.long, device=dev).scatter_add_(0, torch.where(table >= 0, table, torch.full_like(table, P)).reshape(-1), delta.expand_as(table).reshape(-1))
    ref = s["ref"] + flat[:P].to(torch.int32)
    last = (lens[from_] // PAGE).clamp(max=MP - 1)
    partial = torch.gather(rows, 1, last[:, None])[:, 0]
    wants = (parent >= 0) & ~first & (lens[from_] % PAGE > 0) & (partial >= 0)
    got, ref = _lowest_free(ref, wants)
    new.scatter_(1, last[:, None], torch.where(wants, got, torch.gather(new, 1, last[:, None])[:, 0])[:, None])
    src = torch.where(wants & (got >= 0), partial, torch.full_like(partial, -1))
    _plain_copy(s, src, got)
    lens_new = torch.where(parent >= 0, lens[from_], torch.zeros_like(lens))
    return [x.to(torch.int32) for x in (new, lens_new, ref, src, got)] + _all_pools(s)


def _plain_turn(s):
    table, ref = s["table"].long(), s["ref"].clone()
    B, MP = table.shape
    P, dev = s["pool"], table.device
    lp = torch.arange(MP, device=dev)
    gone = (lp >= s["first"].long()[:, None]) & (lp < s["end"].long()[:, None]) & (table >= 0)
    drop = torch.zeros(P + 1, dtype=torch.int32, device=dev).scatter_add_(0, torch.where(gone, table, torch.full_like(table, P)).reshape(-1), gone.reshape(-1).int())
    ref = ref - drop[:P]
    table = torch.where(gone, torch.full_like(table, -1), table)
    lens, many = s["lens"].long()[:, None], s["n_new"].long()[:, None]
    wants = (lp >= lens // PAGE) & (lp < (lens + many + PAGE - 1) // PAGE) & (many > 0) & (table < 0)
    got, ref = _lowest_free(ref, wants)
    return [torch.where(wants, got, table).to(torch.int32), ref]


# -------------------------------------------------------------------------------------------- through this package's API
def _handle(s):
    """The cache handle, outputs and workspaces that a program keeps beside its buffers; made on a state's first pass."""
    if "kv" in s:
        return s
    from paper_2502_02770_amd import binding as B
    dev, op = s["table"].device, s["op"]
    i32 = dict(dtype=torch.int32, device=dev)
    s["B"] = B
    if op == "turn":
        s["live_table"], s["live_ref"] = torch.empty_like(s["table"]), torch.empty_like(s["ref"])
    elif op == "fork":
        s["live_ref"] = torch.empty_like(s["ref"])
    pool = s["k"].shape[0] if "k" in s else s["pool"]
    kv = B.make_kv(s["batch"], s["Hq"], s["Hkv"], s["table"].shape[1], pool, s.get("live_table", s["table"]), s["lens"], s.get("k"), s.get("v"),
                   s.get("codes"), s.get("meta"), s.get("bounds"), quant_bits=s["bits"])
    if op in ("tree", "window"):
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=dev)
        s["ws"] = torch.empty(B.twilight_workspace_bytes(B.TW_WS_NEW_TOKENS, kv, s["max_new"], 0), dtype=torch.uint8, device=dev)
    if op == "fork":
        s["new_table"], s["new_lens"] = torch.empty_like(s["table"]), torch.empty_like(s["lens"])
        s["src"], s["dst"] = torch.empty(s["batch"], **i32), torch.empty(s["batch"], **i32)
    if op in ("fork", "turn"):
        s["status"] = torch.zeros(1, **i32)
        s["ws"] = torch.empty(B.twilight_workspace_bytes(B.TW_WS_PAGES, kv, s.get("max_new", 0), s["batch"]), dtype=torch.uint8, device=dev)
    s["kv"] = kv
    return s


def _run_own(s):
    s = _handle(s)
    B, kv, op = s["B"], s["kv"], s["op"]
    if op == "tree":
        B.twilight_tree_attention(kv, s["q"], s["n_new"], s["offsets"], s["max_new"], s["mask"], s["mask"].shape[1], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "window":
        B.twilight_window_attention(kv, s["q"], s["n_new"], s["offsets"], s["max_new"], s["window"], s["sinks"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "accept":
        B.twilight_pages_copy(kv, s["src"], s["dst"], s["src"].numel())
        B.twilight_tokens_compact(kv, s["keep"], s["count"], s["keep"].shape[1], s["start"], None)
        return _all_pools(s)
    if op == "evict":
        B.twilight_tokens_compact(kv, s["keep"], s["count"], s["keep"].shape[1], s["start"], s["to"])
        return _all_pools(s)
    if op == "fork":
        s["live_ref"].copy_(s["ref"])
        B.twilight_pages_fork(kv, s["parent"], s["batch"], s["new_table"], s["new_lens"], s["live_ref"], s["src"], s["dst"], s["status"], s["ws"])
        B.twilight_pages_copy(kv, s["src"], s["dst"], s["batch"])
        return [s["new_table"], s["new_lens"], s["live_ref"], s["src"], s["dst"]] + _all_pools(s)
    s["live_table"].copy_(s["table"])
    s["live_ref"].copy_(s["ref"])
    B.twilight_pages_free(kv, s["first"], s["end"], s["live_ref"], s["status"])
    B.twilight_pages_reserve(kv, s["n_new"], s["max_new"], s["live_ref"], s["status"], s["ws"])
    return [s["live_table"], s["live_ref"]]


# ------------------------------------------------------------------------------------------- the definition, in 64 bits
def _exact_pages(case, seed):
    """The pools after the moves, one page or sequence at a time."""
    s = prepare(case, seed)
    k, v, codes, meta, bounds = was = [s[n].double() if s[n].is_floating_point() else s[n].clone() for n in ("k", "v", "codes", "meta", "bounds")]
    if case["op"] == "fork":
        table, lens, parent = (s[n].cpu().tolist() for n in ("table", "lens", "parent"))
        held = [0] * s["pool"]
        later, children = [], set()
        for i, r in enumerate(parent):
            if r < 0:
                continue
            own_pages, again = [p for p in table[r] if p >= 0], r in children
            children.add(r)
            whole = lens[r] // PAGE
            for p in own_pages[:whole] if again else own_pages:
                held[p] += 1
            if again and lens[r] % PAGE:
                later.append(table[r][whole])
        free = (p for p in range(s["pool"]) if not held[p])
        for p in later:
            to = next(free, -1)
            if to >= 0:
                for x in was:
                    x[to] = x[p]
        return [None] * 5 + was
    if case["op"] == "accept":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            for x in was:
                x[b] = x[a]
    before = [x.clone() for x in was[:4]]
    for b in range(case["batch"]):
        n, at = int(s["count"][b]), int(s["start"][b])
        a, z = s["keep"][b, :n].long(), torch.arange(at, at + n, device="cuda")
        frm, to = s["table"][b].long(), s["to" if case["op"] == "evict" else "table"][b].long()
        for x, y in zip(was, before):
            x[to[z // PAGE], :, z % PAGE] = y[frm[a // PAGE], :, a % PAGE]
        pages, full = to[at // PAGE:(at + n - 1) // PAGE + 1], (at + n) % PAGE
        bounds[pages] = torch.stack([k[pages].amin(2), k[pages].amax(2)], 2)
        if full:
            bounds[pages[-1]] = torch.stack([k[pages[-1], :, :full].amin(1), k[pages[-1], :, :full].amax(1)], 1)
    return was


def exact(case, seed):
    """Attention from its definition, one sequence, one KV head and some new tokens at a time; the pools as the moves leave
    them.  (Tables and counts are whole numbers, without a rounded value.)"""
    if case["op"] == "turn":
        return None
    if case["op"] not in ("tree", "window"):
        return _exact_pages(case, seed)
    lens, many = _lens(case)
    if sum(_visible(case, n, m)[1] for n, m in zip(lens, many)) * case["q_heads"] > 1.5e10:
        return None
    s = prepare(case, seed)
    hq, hkv, G = case["q_heads"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(sum(many), hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(many), hq), -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, m) in enumerate(zip(lens, many)):
        if not m:
            continue
        pages = s["table"][b, :-(-n // PAGE)].long()
        t = torch.arange(n, device="cuda")
        for h in range(hkv):
            k = s["k"][pages, h].reshape(-1, D)[:n].double()
            v = s["v"][pages, h].reshape(-1, D)[:n].double()
            for i0 in range(0, m, 1024):
                i1 = min(m, i0 + 1024)
                q = s["q"][row + i0:row + i1, h * G:(h + 1) * G].double()                    # [rows, G, D]
                x = (q.reshape(-1, D) @ k.T).reshape(i1 - i0, G, n) / math.sqrt(D)
                if case["op"] == "tree":
                    w = s["mask"][row + i0:row + i1].cpu().numpy()
                    bits = np.unpackbits(np.ascontiguousarray(w).view(np.uint8), axis=1, bitorder="little")[:, :m].astype(bool)
                    hidden = torch.zeros(i1 - i0, n, dtype=torch.bool, device="cuda")
                    hidden[:, n - m:] = ~torch.from_numpy(bits).cuda()
                else:
                    p = torch.arange(n - m + i0, n - m + i1, device="cuda")[:, None]
                    hidden = (t > p) | ((t <= p - case["window"]) & (t >= case["sinks"]))
                x[hidden[:, None].expand_as(x)] = -math.inf
                ls = torch.logsumexp(x, -1)
                w = torch.exp(x - torch.where(ls == -math.inf, torch.zeros_like(ls), ls)[..., None])
                out[row + i0:row + i1, h * G:(h + 1) * G] = (w.reshape(-1, n) @ v).reshape(i1 - i0, G, D)
                lse[row + i0:row + i1, h * G:(h + 1) * G] = ls
        row += m
    return {"out": out, "lse": lse}
