"""Caches in 4 bits for the tests: codes, (scale, zero) and the values they stand for, made without the library."""
import math

import numpy as np
import torch


def unpack(packed):
    """u8 [..., 64] -> codes [..., 128] float64: byte k of word w has dim 8 w + k low, dim 8 w + k + 4 high."""
    c = packed.reshape(*packed.shape[:-1], 16, 1, 4)
    return torch.cat([c & 15, c >> 4], -2).reshape(*packed.shape[:-1], 128).double()


def values(packed, meta):
    """Codes and (scale, zero) -> float64 rows, exact."""
    m = meta.double().repeat_interleave(32, -2)
    return unpack(packed) * m[..., 0] + m[..., 1]


class Cache4:
    """Random codes and (scale, zero) in shuffled pages; what is no token, and pages that no table names, have NaN for (scale, zero)."""

    def __init__(self, lens, hq, hkv, seed=0, max_pages=None, spare=3, shift=0, spread=0.15, mean=-1.0):
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
        self.pools = []
        for _ in range(2):
            codes = torch.randint(0, 256, (P, hkv, 16, 64), device="cuda", dtype=torch.uint8, generator=g)
            meta = torch.stack([spread * (0.2 + torch.rand(P, hkv, 16, 4, device="cuda", generator=g)),
                                mean * (0.5 + torch.rand(P, hkv, 16, 4, device="cuda", generator=g))], -1).half()
            self.pools.append((codes, meta))
        token = torch.zeros(P, 16, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            for i, p in enumerate(self.table[b, :held[b]].tolist()):
                token[p, :min(16, n - 16 * i)] = True
        for _, meta in self.pools:
            meta[~token[:, None, :, None, None].expand_as(meta)] = math.nan
        (self.kc, self.km), (self.vc, self.vm) = self.pools
        self.seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.kv = T.make_kv(len(lens), hq, hkv, self.max_pages, P, self.table, self.seq, None, None, self.kc, self.km)
        self.unmapped = {}

    def unmap(self, b, page, value=-1):
        """Takes a page away: nobody sees its tokens."""
        self.table[b, page] = value
        self.unmapped.setdefault(b, set()).update(range(page * 16, page * 16 + 16))

    def rows(self, which, b, h):
        """float64 rows of K (0) or V (1) of a sequence's head, 0 for those on pages that are not there."""
        n = self.lens[b]
        pages = self.table[b, :-(-n // 16)].long()
        ok = (pages >= 0) & (pages < self.kc.shape[0])
        codes, meta = self.pools[which]
        p = pages.clamp(0, self.kc.shape[0] - 1)
        x = torch.where(ok[:, None, None], values(codes[p, h], meta[p, h]), torch.zeros((), dtype=torch.float64, device="cuda"))
        return x.reshape(-1, 128)[:n]

    def bands(self, b, h):
        """(|scale|, |zero|) of K per dim, [n, 128] each."""
        n = self.lens[b]
        pages = self.table[b, :-(-n // 16)].long().clamp(0, self.kc.shape[0] - 1)
        m = torch.nan_to_num(self.km[pages, h]).double().abs().reshape(-1, 4, 2)[:n].repeat_interleave(32, 1)
        return m[..., 0], m[..., 1]

    def see(self, b, m, window, sinks):
        """[m, len] truth values: what each new token sees."""
        n = self.lens[b]
        t, p = torch.arange(n, device="cuda"), torch.arange(n - m, n, device="cuda")[:, None]
        s = (t <= p) & ((p - t < window) | (t < sinks))
        for x in self.unmapped.get(b, ()):
            if x < n:
                s[:, x] = False
        return s
