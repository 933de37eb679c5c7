"""Refusals of the paged cache's calls and of the projection with epilogue, on
the host: fake, aligned, non-overlapping addresses that are never dereferenced,
and the binding's own checks."""

import os

import pytest
import torch

import paper_2607_16339_amd as lc
from paper_2607_16339_amd import _lib

OK, INVALID, UNSUP = _lib.LACACHE_OK, _lib.LACACHE_ERR_INVALID_ARG, _lib.LACACHE_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return _lib.lib()


def _addr(i):
    return 0x10000000000 + i * (1 << 36)


def _call(fn, names, values, over):
    a = dict(zip(names, values))
    assert set(over) <= set(a), over
    a.update(over)
    return fn(None, *a.values())


def _append(L, **over):
    names = ("qkv seq pos T cos sin rope_len rope_dim table S max_pages q k v ks vs num_pages page heads kv d "
             "kind").split()
    values = [_addr(1), _addr(2), _addr(3), 4, _addr(4), _addr(5), 100, 128, _addr(6), 2, 8, _addr(7), _addr(8), _addr(9),
              None, None, 40, 16, 32, 8, 128, 0]
    return _call(L.lacache_paged_append, names, values, over)


def test_append_refusals(L):
    assert _append(L, T=0) == OK and _append(L, S=0) == OK
    for bad in (dict(T=-1), dict(S=-1), dict(kv=0), dict(heads=0), dict(heads=12), dict(rope_dim=24), dict(rope_dim=144),
                dict(rope_dim=-16), dict(rope_len=0), dict(max_pages=0), dict(num_pages=0), dict(page=0), dict(kind=2),
                dict(kind=-1), dict(d=0), dict(q=None), dict(k=None), dict(seq=None), dict(cos=None), dict(table=None),
                dict(qkv=_addr(1) + 8), dict(q=_addr(1) + 1024), dict(k=_addr(8), v=_addr(8) + 4096),
                dict(q=_addr(6)), dict(k=_addr(2)), dict(v=_addr(5) + 256),
                dict(ks=_addr(10)),                                   # scales beside a bf16 cache
                dict(kind=1), dict(kind=1, ks=_addr(10)),             # an e4m3 cache without its scales
                dict(kind=1, ks=_addr(10), vs=_addr(10)),
                dict(kind=1, ks=_addr(10), vs=_addr(9) + 64)):
        assert _append(L, **bad) == INVALID, bad
    for bad in (dict(d=96), dict(d=256, rope_dim=128), dict(page=8), dict(page=48), dict(page=512), dict(S=4097),
                dict(max_pages=(1 << 18) + 1), dict(num_pages=1 << 31), dict(T=(1 << 24) + 1),
                dict(T=1 << 24), dict(heads=4096, kv=8)):
        assert _append(L, **bad) == UNSUP, bad
    assert _append(L, T=0, rope_dim=0, cos=None, sin=None, rope_len=0) == OK


def _attn(L, fn="lacache_paged_attention", extra=(), **over):
    names = "q k v ks vs table lens o lse S nq heads kv d num_pages page max_pages scale causal kind".split()
    values = [_addr(1), _addr(2), _addr(3), None, None, _addr(4), _addr(5), _addr(6), _addr(7), 2, 1, 32, 8, 128, 40, 16, 8,
              0.1, 1, 0]
    a = dict(zip(names, values))
    assert set(over) <= set(a), over
    a.update(over)
    return getattr(L, fn)(None, *a.values(), *extra)


ATTN_INVALID = (dict(S=-1), dict(nq=0), dict(nq=-1), dict(heads=0), dict(kv=0), dict(heads=30), dict(num_pages=0),
                dict(page=0), dict(max_pages=0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(causal=2), dict(kind=2), dict(q=None), dict(k=None), dict(table=None), dict(lens=None), dict(o=None),
                dict(lse=_addr(7) + 4), dict(o=_addr(1)), dict(o=_addr(2) + 1024), dict(o=_addr(4)), dict(lse=_addr(6)),
                dict(lse=_addr(1)), dict(lse=_addr(5)), dict(ks=_addr(9)), dict(kind=1), dict(kind=1, vs=_addr(9)),
                dict(kind=1, ks=_addr(9), vs=_addr(10) + 8), dict(kind=1, ks=_addr(9), vs=_addr(10), o=_addr(10)))
ATTN_UNSUP = (dict(nq=65), dict(d=96), dict(d=256), dict(page=1), dict(page=24), dict(page=512), dict(S=4097),
              dict(heads=8192), dict(max_pages=(1 << 18) + 1), dict(num_pages=1 << 31),
              dict(S=4096, heads=4096, kv=4096), dict(S=4096, heads=2056, kv=2056), dict(S=4096, nq=64, heads=1032, kv=8))


def test_attention_refusals(L):
    assert _attn(L, S=0) == OK and _attn(L, S=0, q=None) == OK
    for bad in ATTN_INVALID:
        assert _attn(L, **bad) == INVALID, bad
    for bad in ATTN_UNSUP:
        assert _attn(L, **bad) == UNSUP, bad


def test_attention_workspace_refusals(L):
    need = L.lacache_paged_attention_workspace_bytes(2, 1, 32, 8, 128)
    ws = lambda p, n: dict(fn="lacache_paged_attention_ws", extra=(p, n))  # noqa: E731
    assert need > 0
    assert _attn(L, S=0, **ws(None, 0)) == OK
    for p, n in ((None, need), (_addr(9) + 128, need), (_addr(9), need - 1), (_addr(6), need), (_addr(2), need),
                 (_addr(4), need), (_addr(7), need)):
        assert _attn(L, **ws(p, n)) == INVALID, (p, n)
    for bad in ATTN_INVALID:
        assert _attn(L, **ws(_addr(9) + (1 << 35), 1 << 34), **bad) == INVALID, bad
    for bad in ((-1, 1, 32, 8, 128), (2, 0, 32, 8, 128), (2, 65, 32, 8, 128), (2, 1, 30, 8, 128), (2, 1, 32, 8, 96),
                (4097, 1, 32, 8, 128), (2, 1, 0, 0, 128),
                (4096, 1, 4096, 4096, 64)):
        assert L.lacache_paged_attention_workspace_bytes(*bad) == 0, bad


def _linear(L, **over):
    names = "a w bias residual out M N K act".split()
    values = [_addr(1), _addr(2), _addr(3), _addr(4), _addr(5), 16, 256, 128, 0]
    return _call(L.lacache_linear_act_bf16, names, values, over)


def test_linear_act_refusals(L):
    assert _linear(L, M=0) == OK
    for bad in (dict(M=-1), dict(N=100), dict(K=0), dict(K=64), dict(act=6), dict(act=-1), dict(a=None), dict(w=None),
                dict(out=None), dict(bias=_addr(3) + 2), dict(residual=_addr(4) + 8), dict(out=_addr(1)),
                dict(out=_addr(2) + 1024), dict(out=_addr(3)), dict(residual=_addr(5) + 16), dict(residual=_addr(5) - 16)):
        assert _linear(L, **bad) == INVALID, bad
    for bad in (dict(M=(1 << 24) + 1), dict(N=131072 + 128), dict(K=131072 + 128), dict(N=32768, K=32768, act=5)):
        assert _linear(L, **bad) == UNSUP, bad
    # the gate and up rows: twice N
    assert _linear(L, act=5, out=_addr(2) + 256 * 128 * 2 + 4096) == INVALID
    assert _linear(L, M=0, act=5) == OK
    import ctypes
    t = (ctypes.c_int * 2)()
    assert L.lacache_linear_act_tile(300, 256, 128, 0, t) == OK and t[0] in (32, 64, 128, 256) and t[1] in (64, 128, 256)
    for bad in ((0, 256, 128, 0, t), (300, 100, 128, 0, t), (300, 256, 128, 6, t), (300, 256, 128, 0, None)):
        assert L.lacache_linear_act_tile(*bad) == INVALID, bad


def test_binding_refusals():
    """Wrong shapes, types and places are named before the library is called (host tensors: no GPU here)."""
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i32 = torch.int32
    with pytest.raises(ValueError, match="device tensor"):
        lc.lacache_linear_act_bf16(z(4, 128), z(128, 128), z(4, 128), stream=0)
    k, q = z(4, 2, 16, 64), z(2, 1, 4, 64)
    with pytest.raises(ValueError):
        lc.lacache_paged_attention(q, k, k, z(2, 3, dt=i32), z(2, dt=i32), z(2, 1, 4, 64), stream=0)
    with pytest.raises(ValueError, match="num_pages"):
        lc.lacache_paged_attention(q, z(4, 2, 16), k, z(2, 3, dt=i32), z(2, dt=i32), q, stream=0)
    with pytest.raises(ValueError, match="e4m3"):
        lc.lacache_paged_attention(q, k, k, z(2, 3, dt=i32), z(2, dt=i32), q, k_scale=z(4, 2, 16, dt=torch.float32),
                                   stream=0)
    with pytest.raises(ValueError):
        lc.lacache_paged_append(z(2, 8 * 64), z(2, dt=i32), z(2, dt=i32), None, None, z(1, 3, dt=i32), z(2, 4, 64), k, k,
                                stream=0)
