"""Cases for timing the operators of a cache that runs short of memory - K and V held in 4 bits, tokens given up by the
attention they got - and those operators in plain torch.

  store   new rows of K and V quantised into the pages of a 4-bit cache, and read back as bf16 rows
  kv4     attention of the newest tokens of a sequence (one, a draft, a chunk) over a cache held in 4 bits
  mass    the attention weight that every cached token got from the newest tokens, added to what it had
  keep    the tokens with the most accumulated weight picked, first and latest ones always, and their weights packed

The cache is the paged one of this package: pages of 16 tokens, head_dim 128, codes of 4 bits with an fp16 (scale, zero) per
32 dims, x ~ code * scale + zero, for K and, laid out alike, for V; bf16 K where the mass is taken from a bf16 cache.
"""
import math
import random

import numpy as np
import torch

own = False

D, PAGE, GROUP, LEVELS = 128, 16, 32, 15
SCALE = 1.0 / math.sqrt(D)
NO_WINDOW = 2**31 - 1


# ---------------------------------------------------------------------------------------------------------------- cases
def _case(name, op, batch, tokens, new=1, q_heads=32, kv_heads=8, ragged=False, window=NO_WINDOW, sinks=0, codes=True, decay=1.0,
          keep=0.5, recent=0, lens_seed=0):
    c = dict(op=op, batch=batch, tokens=tokens, new=new, q_heads=q_heads, kv_heads=kv_heads, ragged=ragged, window=window, sinks=sinks,
             codes=codes, decay=decay, keep=keep, recent=recent, lens_seed=lens_seed)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a decode step's rows of a serving batch
        _case("store_64x1", "store", 64, 1000, 1, ragged=True, lens_seed=3),
        # prompts on their way into the cache
        _case("store_4x8k", "store", 4, 8192, 8192),
        # one chat's next token: launch and dependency latency
        _case("kv4_1x4k", "kv4", 1, 4096),
        # the ordinary serving batch of long contexts
        _case("kv4_8x32k", "kv4", 8, 32768),
        # mixed traffic of odd lengths on a wide model, single tokens and drafts of up to 7
        _case("kv4_ragged64_g8", "kv4", 64, 32001, 7, q_heads=64, ragged=True, lens_seed=5),
        # chunked prefill behind contexts of odd lengths
        _case("kv4_chunk_odd", "kv4", 3, 9001, 257, window=6001, sinks=4),
        # a chat's step, bf16 K
        _case("mass_1x4k", "mass", 1, 4096, codes=False),
        # the serving batch's step over 4-bit K, older weight fading
        _case("mass_8x32k_codes", "mass", 8, 32768, decay=0.98),
        # the last tokens of long prompts of odd lengths say which of the prompt is worth its place
        _case("mass_last64_odd", "mass", 2, 16001, 64, codes=False),
        # a chat over its budget by a step
        _case("keep_1x2k", "keep", 1, 2049, keep=0.999, sinks=4, recent=256),
        # a serving batch cut to a quarter
        _case("keep_16x32k", "keep", 16, 32768, ragged=True, keep=0.25, sinks=4, recent=512, lens_seed=9),
        # a few very long contexts halved
        _case("keep_3x200k", "keep", 3, 200003, keep=0.5, sinks=16, recent=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["store", "kv4", "kv4", "kv4", "mass", "mass", "keep", "keep"])
    seed = rng.randrange(1 << 30)
    if op == "store":
        kv_heads = rng.choice([8, 8, 4, 32])
        batch = _log_int(rng, 1, 64)
        return _case(None, op, batch, _log_int(rng, 20, max(20, min(8192, (1 << 18) // kv_heads // batch))), _log_int(rng, 1, max(1, min(8192, (1 << 18) // kv_heads // batch))),
                     kv_heads, kv_heads, ragged=rng.random() < 0.6, lens_seed=seed)
    if op == "keep":
        batch = _log_int(rng, 1, 32)
        return _case(None, op, batch, _log_int(rng, 100, min(200000, 600000 // batch)), ragged=rng.random() < 0.5, keep=rng.choice([0.05, 0.25, 0.5, 0.9, 0.999]),
                     sinks=rng.choice([0, 1, 4, 16]), recent=_log_int(rng, 1, 1024), lens_seed=seed)
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (64, 8), (32, 32), (16, 8)])
    batch = _log_int(rng, 1, 48 if op == "kv4" else 16)
    new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 256)])
    # rows of the cache, and scores, of the largest listed cases
    top = min((1 << 21) // kv_heads, (1 << 27) // (new * q_heads)) // batch
    window = rng.choice([NO_WINDOW, NO_WINDOW, _log_int(rng, 64, 8192)])
    return _case(None, op, batch, _log_int(rng, 300, max(400, min(65536, top))), new, q_heads, kv_heads, ragged=rng.random() < 0.5, window=window,
                 sinks=rng.choice([0, 1, 4, 16, 64]) if window < NO_WINDOW else 0, codes=op == "kv4" or rng.random() < 0.5,
                 decay=rng.choice([1.0, 0.98, 0.5]), lens_seed=seed)


def _lens(case):
    """Tokens of each sequence, and how many of them are new."""
    n, b, new = case["tokens"], case["batch"], case["new"]
    if not case["ragged"]:
        return [n] * b, [min(new, n)] * b
    r = random.Random(case["lens_seed"])
    lens = [_log_int(r, max(1, n // 32), n) for _ in range(b)]
    many = [min(x, r.choice([new, new, r.randint(1, new), 1])) for x in lens]
    lens[0], many[0] = n, min(new, n)
    return lens, many


def _seen(case, n, new):
    """(positions that any of the new tokens sees, pairs of a new token and a position) of a sequence."""
    p = np.arange(n - new, n, dtype=np.int64)
    sinks = np.minimum(case["sinks"], np.maximum(0, p + 1 - case["window"]))
    first = max(0, n - new - case["window"] + 1)
    return n - first + min(case["sinks"], first), int((np.minimum(case["window"], p + 1) + sinks).sum())


def work(case):
    op, hq, hkv = case["op"], case["q_heads"], case["kv_heads"]
    lens, many = _lens(case)
    code = D // 2 + 4 * D // GROUP                                   # a row in 4 bits
    if op == "store":
        rows = sum(many) * hkv
        return {"bytes": rows * 2.0 * (2 * D * 2 + 2 * code), "flops": 0.0}
    if op == "keep":
        kept = sum(max(1, int(case["keep"] * n)) for n in lens)
        return {"bytes": 4.0 * sum(lens) + 8.0 * kept, "flops": 0.0}
    seen = [_seen(case, n, m) for n, m in zip(lens, many)]
    rows, pages = sum(many) * hq, sum(-(-n // PAGE) for n in lens) * 4
    if op == "kv4":
        return {"bytes": sum(s[0] for s in seen) * hkv * 2.0 * code + rows * (2 * D * 2 + 4) + pages, "flops": 4.0 * D * hq * sum(s[1] for s in seen)}
    return {"bytes": sum(s[0] for s in seen) * hkv * (code if case["codes"] else 2.0 * D) + rows * (D * 2 + 4) + pages + 8.0 * sum(lens),
            "flops": 2.0 * D * hq * sum(s[1] for s in seen)}


# --------------------------------------------------------------------------------------------------------------- inputs
def _i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()


def _table(lens, max_pages, rng):
    """Pages of all sequences in shuffled order; [batch, max_pages], -1 beyond a sequence's pages."""
    held = [-(-n // PAGE) for n in lens]
    ids = rng.permutation(sum(held))
    table = np.full((len(lens), max_pages), -1, dtype=np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    return table, sum(held)


def _quantise(x):
    """Rows [..., 128] -> (codes [..., 128] as numbers, (scale, zero) fp16 [..., 4, 2]), one fp32 operation after the other."""
    g = x.float().unflatten(-1, (D // GROUP, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    scale, zero = ((hi - lo) * np.float32(1 / LEVELS).item()).half(), lo.half()
    inv = (1.0 / scale.double()).float()
    c = torch.clamp(torch.round((g - zero.float()[..., None]) * inv[..., None]), 0, LEVELS)
    c = torch.where(scale[..., None] == 0, torch.zeros_like(c), c)
    return c.flatten(-2), torch.stack([scale, zero], -1)


def _values(codes, meta):
    m = meta.float()
    return (codes.unflatten(-1, (D // GROUP, GROUP)) * m[..., 0, None] + m[..., 1, None]).flatten(-2)


def _pack(codes):
    """[..., 128] -> u8 [..., 64]: byte k of word w holds the code of dim 8 w + k low, that of 8 w + k + 4 high."""
    c = codes.to(torch.uint8).unflatten(-1, (16, 2, 4))
    return (c[..., 0, :] | c[..., 1, :] << 4).flatten(-2)


def _unpack(packed):
    c = packed.unflatten(-1, (16, 1, 4))
    return torch.cat([c & 15, c >> 4], -2).flatten(-3).float()


def _four_bits(P, hkv, g, mean):
    """A pool of quantised rows -> (packed codes, (scale, zero)), some thousand pages at a time."""
    codes = torch.empty(P, hkv, PAGE, D // 2, dtype=torch.uint8, device="cuda")
    meta = torch.empty(P, hkv, PAGE, D // GROUP, 2, dtype=torch.float16, device="cuda")
    for i in range(0, P, 4096):
        c, meta[i:i + 4096] = _quantise(torch.randn(min(4096, P - i), hkv, PAGE, D, device="cuda", generator=g) + mean)
        codes[i:i + 4096] = _pack(c)
    return codes, meta


def _queries(rows, hq, g):
    """Queries of different sharpness, from even to peaked attention."""
    return (torch.randn(rows, hq, D, device="cuda", generator=g) * (0.5 + 2.5 * torch.rand(1, hq, 1, device="cuda", generator=g))).to(torch.bfloat16)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    op, hq, hkv, B = case["op"], case["q_heads"], case["kv_heads"], case["batch"]
    lens, many = _lens(case)
    s = dict(op=op, Hq=hq, Hkv=hkv, batch=B, max_new=case["new"], window=case["window"], sinks=case["sinks"])
    if op == "keep":
        max_pages = -(-max(lens) // PAGE)
        # weights as they come together over many steps: a few tokens have most, those that no token sees any more have none
        mass = torch.exp(2.5 * torch.randn(B, max_pages * PAGE, device="cuda", generator=g) - 4)
        mass = torch.where(torch.rand(mass.shape, device="cuda", generator=g) < 0.1, torch.zeros_like(mass), mass)
        budget = [max(1, int(case["keep"] * n)) for n in lens]
        s.update(mass=mass, lens=_i32(lens), budget=_i32(budget), stride=max(budget), recent=case["recent"], max_pages=max_pages,
                 table=_i32(np.zeros((B, max_pages))))
        return s
    offsets = np.cumsum([0] + many[:-1])
    full = [n + m for n, m in zip(lens, many)] if op == "store" else lens
    table, P = _table(full, -(-max(full) // PAGE), rng)
    s.update(table=_i32(table), lens=_i32(lens), n_new=_i32(many), offsets=_i32(offsets), rows=sum(many), pool=P)
    if op == "store":
        # rows with channels of their own mean and spread, as a layer's keys and values have
        for n in ("k", "v"):
            mean, spread = torch.randn(1, hkv, D, device="cuda", generator=g), 0.3 + torch.rand(1, hkv, D, device="cuda", generator=g)
            s[n + "_new"] = (mean + spread * torch.randn(sum(many), hkv, D, device="cuda", generator=g)).to(torch.bfloat16)
            s[n + "_codes"], s[n + "_meta"] = _four_bits(P, hkv, g, 0.0)
        s["bounds"] = torch.stack([torch.full((P, hkv, D), -0.25, device="cuda"), torch.full((P, hkv, D), 0.25, device="cuda")], 2).to(torch.bfloat16)
        return s
    s["q"] = _queries(sum(many), hq, g)
    if op == "kv4" or case["codes"]:
        s["k_codes"], s["k_meta"] = _four_bits(P, hkv, g, 0.0)
    else:
        s["k"] = torch.randn(P, hkv, PAGE, D, device="cuda", dtype=torch.bfloat16, generator=g)
    if op == "kv4":
        s["v_codes"], s["v_meta"] = _four_bits(P, hkv, g, 0.5)
        return s
    x, _ = _scores(s)
    top = x.amax(-1, keepdim=True)
    s["lse"] = _to_rows(s, (top + x.sub_(top).exp_().sum(-1, keepdim=True).log())[..., 0]).contiguous()
    s["mass"] = torch.rand(B, table.shape[1] * PAGE, device="cuda", generator=g)
    s["decay"] = case["decay"]
    return s


# ------------------------------------------------------------------------------------------------------- the operators
def run(state):
    if own:
        return _run_own(state)
    return dict(store=_plain_store, kv4=_plain_kv4, mass=_plain_mass, keep=_plain_keep)[state["op"]](state)


def _where(s):
    """Sequence, position, page and slot of every new row; store's new rows follow the sequence's tokens."""
    many = s["n_new"].long()
    b = torch.repeat_interleave(torch.arange(s["batch"], device=many.device), many, output_size=s["rows"])
    p = s["lens"].long()[b] + torch.arange(s["rows"], device=many.device) - s["offsets"].long()[b]
    return b, p, s["table"].long()[b, p // PAGE], p % PAGE


def _plain_store(s):
    b, p, page, slot = _where(s)
    out = {}
    for n in ("k", "v"):
        codes, meta = _quantise(s[n + "_new"])
        s[n + "_codes"][page, :, slot] = _pack(codes)
        s[n + "_meta"][page, :, slot] = meta
        out[n] = _values(codes, meta).to(torch.bfloat16)
        out[n + "_meta"] = s[n + "_meta"]
    # bounds: of a page that held tokens already joined with theirs, of others those of the new rows
    rows, old = s["k_new"].float(), s["bounds"].float()
    begun = torch.zeros(s["pool"] + 1, dtype=torch.bool, device=page.device)
    held = s["lens"].long()
    last = torch.gather(s["table"].long(), 1, (held // PAGE).clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0]
    begun[torch.where(held % PAGE > 0, last, torch.full_like(last, s["pool"]))] = True
    fresh = torch.zeros(s["pool"], dtype=torch.bool, device=page.device)
    fresh[page] = True
    fresh = (fresh & ~begun[:-1])[:, None, None]
    lo = torch.where(fresh, torch.full_like(old[:, :, 0], math.inf), old[:, :, 0])
    hi = torch.where(fresh, torch.full_like(old[:, :, 1], -math.inf), old[:, :, 1])
    at = page[:, None, None].expand_as(rows)
    lo.scatter_reduce_(0, at, rows, "amin")
    hi.scatter_reduce_(0, at, rows, "amax")
    s["bounds"].copy_(torch.stack([lo, hi], 2).to(torch.bfloat16))
    out["bounds"] = s["bounds"]
    return out


def _rows_of(s, name):
    """fp32 rows of K or V, [B, Hkv, L, 128]."""
    pages = s["table"].long().clamp(min=0)
    x = _values(_unpack(s[name + "_codes"][pages]), s[name + "_meta"][pages]) if name + "_codes" in s else s[name][pages].float()
    return x.transpose(2, 3).reshape(s["batch"], -1, s["Hkv"], D).transpose(1, 2).contiguous()


def _scores(s):
    """Scaled scores [B, Hkv, G, T, L] of the new tokens, -inf where a token sees nothing; new tokens that a sequence does not
    have see what its last one does."""
    B, Hkv, T = s["batch"], s["Hkv"], s["max_new"]
    G, dev = s["Hq"] // Hkv, s["q"].device
    k = _rows_of(s, "k")
    L = k.shape[2]
    lens, many = s["lens"].long()[:, None, None], s["n_new"].long()[:, None, None]
    i, t = torch.arange(T, device=dev)[:, None], torch.arange(L, device=dev)
    i = torch.minimum(i, many - 1)                                                                        # [B, T, 1]
    p = lens - many + i
    see = (t <= p) & ((p - t < s["window"]) | (t < s["sinks"])) & (t < lens)
    q = s["q"][s["offsets"].long()[:, None] + i[..., 0]].float().view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hkv, G, T, L).mul_(SCALE)
    return x.masked_fill_(~see[:, None, None], -math.inf), L


def _to_rows(s, x):
    """[B, Hkv, G, T, ...] -> [rows, Hq, ...]"""
    r = torch.arange(s["rows"], device=x.device)
    b = torch.searchsorted((s["offsets"].long() + s["n_new"].long()).contiguous(), r, right=True)
    return x.movedim(3, 1).flatten(2, 3)[b, r - s["offsets"].long()[b]]


def _plain_kv4(s):
    x, L = _scores(s)
    m = x.amax(-1, keepdim=True)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(2, 3), _rows_of(s, "v")).view(*x.shape[:4], D) / total
    return {"out": _to_rows(s, o).to(torch.bfloat16), "lse": _to_rows(s, (m + total.log())[..., 0])}


def _plain_mass(s):
    x, L = _scores(s)
    B, T, dev = s["batch"], s["max_new"], x.device
    lens, many = s["lens"].long()[:, None], s["n_new"].long()[:, None]
    i = torch.arange(T, device=dev)
    lse = s["lse"][s["offsets"].long()[:, None] + torch.minimum(i, many - 1)].view(B, T, s["Hkv"], -1).permute(0, 2, 3, 1)
    x.sub_(lse[..., None]).exp_()
    x.masked_fill_((i >= many)[:, None, None, :, None], 0.0)
    got = x.sum((1, 2, 3))
    t = torch.arange(L, device=dev)
    had = torch.where(t < lens - many, s["decay"] * s["mass"], torch.zeros_like(s["mass"]))
    return torch.where(t < lens, had + got, s["mass"])


def _plain_keep(s):
    mass, lens = s["mass"], s["lens"].long()[:, None]
    B, L = mass.shape
    t = torch.arange(L, device=mass.device)
    budget = torch.minimum(s["budget"].long()[:, None], lens).clamp(0, s["stride"])
    sinks = budget.clamp(max=s["sinks"])
    recent = (budget - sinks).clamp(max=s["recent"])
    rank = torch.where((t < sinks) | (t >= lens - recent), torch.full_like(mass, math.inf), mass)
    rank = torch.where(t < lens, rank, torch.full_like(mass, -math.inf))
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices            # ties: the lowest position first
    kept = torch.zeros(B, L + 1, dtype=torch.bool, device=mass.device)
    kept.scatter_(1, torch.where(t < budget, order, torch.full_like(order, L)), True)
    kept = kept[:, :L]
    at = torch.where(kept, torch.cumsum(kept.long(), 1) - 1, torch.full_like(order, s["stride"]))
    idx = torch.full((B, s["stride"] + 1), -1, dtype=torch.int32, device=mass.device)
    idx.scatter_(1, at, t.to(torch.int32).expand(B, L))
    out = torch.zeros(B, s["stride"] + 1, device=mass.device)
    out.scatter_(1, at, mass)
    return {"idx": idx[:, :-1].contiguous(), "count": budget[:, 0].to(torch.int32), "mass": out[:, :-1].contiguous()}


# -------------------------------------------------------------------------------------------- through this package's API
def _handle(s):
    """The cache handle, outputs and workspaces that a program keeps beside its buffers; made on a state's first pass."""
    if "kv" in s:
        return s
    from paper_2502_02770_amd import binding as B
    dev, op = s["table"].device, s["op"]
    s["B"] = B
    s["kv"] = kv = B.make_kv(s["batch"], s["Hq"], s["Hkv"], s["table"].shape[1], s.get("pool", 1), s["table"], s["lens"], s.get("k"), None,
                             s.get("k_codes"), s.get("k_meta"), s.get("bounds"))
    if op == "store":
        s["k_out"], s["v_out"] = torch.empty_like(s["k_new"]), torch.empty_like(s["v_new"])
        s["after"] = s["lens"] + s["n_new"]
        s["grown"] = B.make_kv(s["batch"], s["Hq"], s["Hkv"], s["table"].shape[1], s["pool"], s["table"], s["after"], None, None, s["k_codes"], s["k_meta"])
    elif op == "kv4":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=dev)
        s["ws"] = torch.empty(B.twilight_workspace_bytes(B.TW_WS_KV4, kv, s["max_new"]), dtype=torch.uint8, device=dev)
    elif op == "mass":
        s["mass_out"] = s["mass"].clone()
    else:
        s["idx"] = torch.full((s["batch"], s["stride"]), -1, dtype=torch.int32, device=dev)
        s["count"] = torch.zeros(s["batch"], dtype=torch.int32, device=dev)
        s["packed"] = torch.zeros(s["batch"], s["stride"], device=dev)
        s["ws"] = torch.empty(B.twilight_workspace_bytes(B.TW_WS_KEEP, kv), dtype=torch.uint8, device=dev)
    return s


def _run_own(s):
    s = _handle(s)
    B, kv, op = s["B"], s["kv"], s["op"]
    if op == "store":
        B.twilight_kv4_append(kv, s["v_codes"], s["v_meta"], s["k_new"], s["v_new"], s["lens"], s["n_new"], s["offsets"], s["max_new"])
        B.twilight_kv4_read(s["grown"], s["v_codes"], s["v_meta"], s["lens"], s["n_new"], s["offsets"], s["max_new"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "k_meta": s["k_meta"], "v": s["v_out"], "v_meta": s["v_meta"], "bounds": s["bounds"]}
    if op == "kv4":
        B.twilight_kv4_attention(kv, s["v_codes"], s["v_meta"], s["q"], s["n_new"], s["offsets"], s["max_new"], s["window"], s["sinks"], s["out"], s["lse"],
                                 s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "mass":
        B.twilight_attention_mass(kv, s["q"], s["lse"], s["n_new"], s["offsets"], s["max_new"], s["window"], s["sinks"], s["decay"], s["mass"], s["mass_out"])
        return s["mass_out"]
    B.twilight_keep_tokens(kv, s["mass"], s["budget"], s["sinks"], s["recent"], s["idx"], s["count"], s["stride"], s["packed"], s["ws"])
    return {"idx": s["idx"], "count": s["count"], "mass": s["packed"]}


# ------------------------------------------------------------------------------------------- the definition, in 64 bits
def _row64(s, name, b, h, n):
    """Rows 0 .. n - 1 of a sequence's K or V for one head."""
    pages = s["table"][b, :-(-n // PAGE)].long()
    if name + "_codes" not in s:
        return s[name][pages, h].reshape(-1, D)[:n].double()
    words = s[name + "_codes"][pages, h].reshape(-1, 16, 4)[:n].long()
    codes = torch.empty(n, 16, 8, dtype=torch.float64, device="cuda")
    codes[:, :, :4], codes[:, :, 4:] = (words % 16).double(), (words // 16).double()
    m = s[name + "_meta"][pages, h].reshape(-1, D // GROUP, 2)[:n].double()
    return codes.view(n, D) * m[:, :, 0].repeat_interleave(GROUP, 1) + m[:, :, 1].repeat_interleave(GROUP, 1)


def _exact_store(case, s):
    """(scale, zero) of the new rows before their rounding, and the bounds; a code next to the border between two has no value
    that a rounded scale would not move by a step."""
    out = dict(k=None, v=None)
    lens, many = _lens(case)
    bounds = s["bounds"].double()
    for n in ("k", "v"):
        meta = s[n + "_meta"].double()
        row = 0
        for b, (at, m) in enumerate(zip(lens, many)):
            x = s[n + "_new"][row:row + m].double()
            p = torch.arange(at, at + m, device="cuda")
            pages = s["table"][b].long()
            for g in range(D // GROUP):
                y = x[:, :, g * GROUP:(g + 1) * GROUP]
                lo, hi = y.min(2).values, y.max(2).values
                meta[pages[p // PAGE], :, p % PAGE, g] = torch.stack([(hi - lo) / LEVELS, lo], 2)
            if n == "k":
                for lp in range(at // PAGE, (at + m - 1) // PAGE + 1):
                    y = x[max(0, lp * PAGE - at):(lp + 1) * PAGE - at]
                    lo, hi = y.min(0).values, y.max(0).values
                    if lp * PAGE < at:
                        lo, hi = torch.minimum(lo, bounds[pages[lp], :, 0]), torch.maximum(hi, bounds[pages[lp], :, 1])
                    bounds[pages[lp]] = torch.stack([lo, hi], 1)
            row += m
        out[n + "_meta"] = meta
    out["bounds"] = bounds
    return out


def _exact_keep(s):
    lens, budget = s["lens"].cpu().numpy(), s["budget"].cpu().numpy()
    mass = s["mass"].double().cpu().numpy()
    packed = np.zeros((s["batch"], s["stride"]))
    for b, n in enumerate(lens):
        k = int(min(budget[b], n, s["stride"]))
        first = min(s["sinks"], k)
        last = min(s["recent"], k - first)
        order = np.lexsort((np.arange(n), -mass[b, :n]))
        order = [t for t in order if first <= t < n - last][:k - first - last]
        kept = sorted(list(range(first)) + order + list(range(n - last, n)))
        packed[b, :k] = mass[b, kept]
    return {"idx": None, "count": None, "mass": torch.from_numpy(packed).cuda()}


def exact(case, seed):
    """Each operator from its definition, one sequence, one KV head and some new tokens at a time.  (Kept positions are whole
    numbers, without a rounded value.)"""
    lens, many = _lens(case)
    if case["op"] in ("kv4", "mass") and sum(_seen(case, n, m)[1] for n, m in zip(lens, many)) * case["q_heads"] > 1.5e10:
        return None
    s = prepare(case, seed)
    if case["op"] == "store":
        return _exact_store(case, s)
    if case["op"] == "keep":
        return _exact_keep(s)
    hq, hkv, G = case["q_heads"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(sum(many), hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(sum(many), hq, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if case["op"] == "mass" else None
    row = 0
    for b, (n, m) in enumerate(zip(lens, many)):
        t = torch.arange(n, device="cuda")
        if mass is not None:
            mass[b, :n - m] *= case["decay"]
            mass[b, n - m:n] = 0
        for h in range(hkv):
            k = _row64(s, "k", b, h, n)
            v = _row64(s, "v", b, h, n) if mass is None else None
            for i0 in range(0, m, 256):
                i1 = min(m, i0 + 256)
                q = s["q"][row + i0:row + i1, h * G:(h + 1) * G].double()                    # [rows, G, D]
                x = (q.reshape(-1, D) @ k.T).reshape(i1 - i0, G, n) / math.sqrt(D)
                p = torch.arange(n - m + i0, n - m + i1, device="cuda")[:, None]
                hidden = (t > p) | ((t <= p - case["window"]) & (t >= case["sinks"]))
                x[hidden[:, None].expand_as(x)] = -math.inf
                if mass is not None:
                    mass[b, :n] += torch.exp(x - s["lse"][row + i0:row + i1, h * G:(h + 1) * G].double()[..., None]).sum((0, 1))
                    continue
                ls = torch.logsumexp(x, -1)
                out[row + i0:row + i1, h * G:(h + 1) * G] = (torch.exp(x - ls[..., None]).reshape(-1, n) @ v).reshape(i1 - i0, G, D)
                lse[row + i0:row + i1, h * G:(h + 1) * G] = ls
        row += m
    return mass if mass is not None else {"out": out, "lse": lse}
