"""The binding of the cache in 4 bits and of tokens given up refuses lists and rows that are too short, before the library reads or writes
behind them (no GPU: tensors of the CPU, and a library that must not be called)."""
import pytest
import torch

from tests.test_new_operators_cpu import T, _kv  # noqa: F401  (a fixture)


@pytest.fixture
def calls(T, monkeypatch):  # noqa: F811
    """Calls that reached the library."""
    B, seen = T.binding, []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: seen.append(name) or 0

    for f in ("_ints", "_rows", "_sums", "_ptr", "_stream_of"):
        monkeypatch.setattr(B, f, lambda t: None)
    monkeypatch.setattr(B, "_v_pools", lambda *args: (None, None))
    monkeypatch.setattr(B, "lib", lambda: Lib())
    return seen


i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
rows = lambda n, h=8: torch.zeros(n, h, 128, dtype=torch.bfloat16)  # noqa: E731


def given(good, bad, call, calls):
    call(**good)
    assert len(calls) == 1
    for name, value in bad:
        with pytest.raises(AssertionError, match="a number per sequence|a row"):
            call(**dict(good, **{name: value}))
    assert len(calls) == 1


SHORT = [("n_new", i32(2)), ("new_offsets", i32(2)), ("lse", torch.zeros(5, 8)), ("lse", torch.zeros(47))]


def test_attention_over_codes(T, calls):  # noqa: F811
    kv, ws = _kv(T, batch=3, hq=8, hkv=8), torch.zeros(4)
    f = lambda q, n_new, new_offsets, max_new, out, lse: T.twilight_kv4_attention(  # noqa: E731
        kv, None, None, q, n_new, new_offsets, max_new, 9, 0, out, lse, ws)
    good = dict(q=rows(6), n_new=i32(3), new_offsets=i32(3), max_new=2, out=rows(6), lse=torch.zeros(6, 8))
    given(good, SHORT + [("out", rows(5)), ("q", rows(7))], f, calls)
    f(**dict(good, lse=None))
    f(**dict(good, n_new=None, new_offsets=None))
    for bad in (dict(q=rows(5)), dict(max_new=3)):                 # a row per new token, max_new of each sequence
        with pytest.raises(AssertionError, match="a row per new token"):
            f(**dict(good, n_new=None, new_offsets=None, **bad))
    with pytest.raises(AssertionError, match="a row per new token"):
        f(**dict(good, n_new=None, max_new=7))


def test_mass(T, calls):  # noqa: F811
    kv, m = _kv(T, batch=3, hq=8, hkv=8, max_pages=4), torch.zeros(3, 64)
    f = lambda q, n_new, new_offsets, max_new, lse: T.twilight_attention_mass(  # noqa: E731
        kv, q, lse, n_new, new_offsets, max_new, 9, 0, 1.0, m, m)
    good = dict(q=rows(6), n_new=i32(3), new_offsets=i32(3), max_new=2, lse=torch.zeros(6, 8))
    given(good, SHORT + [("q", rows(7))], f, calls)
    f(**dict(good, n_new=None, new_offsets=None))
    with pytest.raises(AssertionError, match="a row per new token"):
        f(**dict(good, n_new=None, new_offsets=None, max_new=3))


@pytest.mark.parametrize("read", [False, True])
def test_rows_of_codes(T, calls, read):  # noqa: F811
    kv = _kv(T, batch=3)
    call = T.twilight_kv4_read if read else T.twilight_kv4_append
    f = lambda start, n, off: (call(kv, None, None, start, n, off, 4, rows(9), rows(9)) if read  # noqa: E731
                               else call(kv, None, None, rows(9), rows(9), start, n, off, 4))
    given(dict(start=i32(3), n=i32(3), off=i32(3)), [("start", i32(2)), ("n", i32(1)), ("off", i32(2))], f, calls)
