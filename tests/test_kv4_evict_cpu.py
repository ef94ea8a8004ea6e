"""Host-side refusals and workspace sizes of the cache in 4 bits and of tokens given up (no GPU)."""
import ctypes

import pytest
import torch

from tests.test_kernel_resources_cpu import _fits, kernels  # noqa: F401  (a fixture)
from tests.test_new_operators_cpu import ONE, PLENTY, T, _kv  # noqa: F401  (a fixture)

NONE = 2**31 - 1
ODD = ctypes.c_void_p(4104)


def codes_only(T, **kw):
    kv = _kv(T, **kw)
    kv.k_pool = kv.v_pool = None
    return kv


def test_attention_over_codes_refuses(T):
    L, ref = T.binding.lib(), ctypes.byref
    f = lambda kv=None, vq=ONE, vm=ONE, q=ONE, max_new=8, window=64, sinks=4, out=ONE, ws=ONE, n=PLENTY: L.twilight_kv4_attention(
        ref(kv or codes_only(T)), vq, vm, q, None, None, max_new, window, sinks, out, None, ws, n, None)
    for name in ("vq", "vm", "q", "out"):
        assert f(**{name: None}) == f(**{name: ODD}) == -1
    assert f(max_new=0) == f(max_new=-1) == f(max_new=(1 << 20) + 1) == f(window=0) == f(sinks=-1) == -1
    assert f(ws=None) == f(n=16) == -2 and f(ws=ODD) == -1
    assert f(kv=codes_only(T, bits=8)) == f(kv=codes_only(T, bits=2)) == f(kv=_kv(T, pools=False)) == -1
    assert f(kv=codes_only(T, max_pages=(1 << 24) + 1)) == -1
    assert f(kv=codes_only(T, batch=8000, hq=8, hkv=1), max_new=1 << 20) == -1
    for name in ("kq_pool", "kq_meta"):
        kv = codes_only(T)
        setattr(kv, name, 4104)
        assert f(kv=kv) == -1
        setattr(kv, name, None)
        assert f(kv=kv) == -1


@pytest.mark.parametrize("read", [False, True])
def test_rows_of_codes_refuse(T, read):
    L, ref = T.binding.lib(), ctypes.byref

    def f(kv=None, vq=ONE, vm=ONE, k=ONE, v=ONE, start=ONE, n=ONE, off=ONE, most=4):
        kv = ref(kv or codes_only(T))
        if read:
            return L.twilight_kv4_read(kv, vq, vm, start, n, off, most, k, v, None)
        return L.twilight_kv4_append(kv, vq, vm, k, v, start, n, off, most, None)
    for name in ("vq", "vm", "k", "v"):
        assert f(**{name: None}) == f(**{name: ODD}) == -1
    assert f(start=None) == f(n=None) == f(off=None) == f(most=-1) == f(most=(1 << 27) + 1) == -1
    assert f(most=0) == 0
    assert f(kv=codes_only(T, bits=8)) == f(kv=_kv(T, pools=False)) == f(kv=codes_only(T, max_pages=(1 << 24) + 1)) == -1


def test_mass_refuses(T):
    L, ref = T.binding.lib(), ctypes.byref
    f = lambda kv=None, q=ONE, lse=ONE, max_new=8, window=64, sinks=4, decay=1.0, a=ONE, b=ONE: L.twilight_attention_mass(
        ref(kv or _kv(T)), q, lse, None, None, max_new, window, sinks, ctypes.c_float(decay), a, b, None)
    assert f(q=None) == f(lse=None) == f(a=None) == f(b=None) == f(q=ODD) == -1
    assert f(max_new=0) == f(max_new=(1 << 20) + 1) == f(window=0) == f(sinks=-1) == -1
    assert f(decay=-0.5) == f(decay=float("nan")) == f(decay=float("inf")) == -1
    assert f(kv=_kv(T, max_pages=(1 << 22) + 1)) == f(kv=_kv(T, pools=False)) == -1
    assert f(kv=codes_only(T, bits=8)) == -1                       # without bf16 K, codes of 4 bits
    assert f(kv=_kv(T, batch=8000, hq=8, hkv=1), max_new=1 << 20) == -1


def test_choice_of_tokens_refuses(T):
    L, ref = T.binding.lib(), ctypes.byref
    f = lambda kv=None, mass=ONE, budget=ONE, sinks=4, recent=4, idx=ONE, count=ONE, stride=8, ws=ONE, n=PLENTY: L.twilight_keep_tokens(
        ref(kv or _kv(T)), mass, budget, sinks, recent, idx, count, stride, None, ws, n, None)
    assert f(mass=None) == f(budget=None) == f(idx=None) == f(count=None) == f(mass=ODD) == f(ws=ODD) == -1
    assert f(sinks=-1) == f(recent=-1) == f(stride=0) == f(stride=-5) == f(kv=_kv(T, max_pages=(1 << 24) + 1)) == -1
    assert f(ws=None) == f(n=16) == -2
    assert f(kv=_kv(T, max_pages=4096), n=4096) == -2              # 65536 tokens: histograms of their chunks


def test_workspaces(T):
    size = T.twilight_workspace_bytes
    # single tokens: two places of 16 rows per 256 tokens of a list, as far as the chip has workgroups
    parts = 2 * 8 * (2 * 8) * 16
    assert parts * 520 <= size(T.TW_WS_KV4, _kv(T, max_pages=128), 1) <= parts * 520 + 1024
    assert size(T.TW_WS_KV4, _kv(T, max_pages=1 << 20), 1) == size(T.TW_WS_KV4, _kv(T, max_pages=1 << 22), 1) <= 2 * 512 * 16 * 520 + 1024
    assert size(T.TW_WS_KV4, _kv(T), 0) == size(T.TW_WS_KV4, _kv(T), -3) == 0
    assert size(T.TW_WS_KEEP, _kv(T, max_pages=512)) == 256
    assert 2 * 5 * 5122 * 4 <= size(T.TW_WS_KEEP, _kv(T, max_pages=2049)) <= 2 * 5 * 5122 * 4 + 512
    assert size(T.TW_WS_KEEP, _kv(T, max_pages=1 << 24)) <= 2 * 128 * 5122 * 4 + 512


def test_compaction_of_codes_alone(T):
    L, ref = T.binding.lib(), ctypes.byref
    kv = codes_only(T)
    f = lambda: L.twilight_tokens_compact(ref(kv), ONE, ONE, 4, ONE, None, None)
    assert f() == -1                                               # bounds would need the rows of K
    kv.page_minmax = None
    kv.v_pool = 4096
    assert f() == -1
    kv.v_pool, kv.kq_pool = None, None
    assert f() == -1


def test_the_binding_refuses(T):
    """Shapes and types, before anything reaches the library."""
    B = T.binding
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    f32 = lambda *n: torch.zeros(*n)
    with pytest.raises(AssertionError, match="as large as K's"):    # on the CPU
        B._v_pools(_kv(T), torch.zeros(64, 8, 16, 64, dtype=torch.uint8), torch.zeros(64, 8, 16, 4, 2, dtype=torch.float16))
    kv = _kv(T, batch=3, max_pages=4)
    for bad in (dict(mass_in=f32(3, 32)), dict(mass_out=f32(2, 64))):
        a = dict(mass_in=f32(3, 64), mass_out=f32(3, 64), **{})
        a.update(bad)
        with pytest.raises(AssertionError, match="a weight per position"):
            B.twilight_attention_mass(kv, None, None, None, None, 1, 1, 0, 1.0, a["mass_in"], a["mass_out"])
    good = dict(mass=f32(3, 64), budget=i32(3), idx=i32(3, 9), count=i32(3), stride=9, out=f32(3, 9))
    for bad in (dict(mass=f32(3, 63)), dict(budget=i32(2)), dict(count=i32(4)), dict(idx=i32(3, 8)), dict(out=f32(3, 8))):
        a = dict(good, **bad)
        with pytest.raises(AssertionError):
            B.twilight_keep_tokens(kv, a["mass"], a["budget"], 0, 0, a["idx"], a["count"], a["stride"], a["out"], None)
    m = object.__new__(T.TokenMass)
    c = m.cache = object.__new__(T.PagedKV)
    c.batch, c.kv = 3, kv
    q, lse = torch.zeros(6, 8, 128, dtype=torch.bfloat16), f32(6, 8)
    for bad in (dict(n_new=i32(2)), dict(lse=f32(5, 8)), dict(max_new=3)):
        a = dict(dict(lse=lse, max_new=2, n_new=None), **bad)
        with pytest.raises(AssertionError):
            m.add(q, a["lse"], a["max_new"], n_new=a["n_new"])
    four = object.__new__(T.PagedKV4)
    four.batch, four.kv, four.device = 3, kv, "cpu"
    with pytest.raises(AssertionError):
        four.over(i32(4, 5), i32(3))
    n = object.__new__(T.NewTokens)
    n.cache, n.out = four, q
    with pytest.raises(AssertionError, match="bf16 pools"):
        n.tree(q, i32(6, 1))


def test_kernels_spill_nothing(kernels):  # noqa: F811
    """But for two forms that stride over items: addresses that their loops do not change."""
    new = {n: k for n, k in kernels.items() if n.startswith(("kv4_", "attention_mass", "keep_"))}
    assert len(new) >= 18
    for n, k in new.items():
        assert k[".vgpr_spill_count"] <= {"kv4_attention_kernel<2, true>": 24, "kv4_wide_kernel<true>": 6}.get(n, 0), n
        if n.startswith(("kv4_attention_kernel", "kv4_wide_kernel")):
            assert _fits(k, 2) and k[".group_segment_fixed_size"] * 2 <= 160 * 1024, (n, k[".vgpr_count"])
