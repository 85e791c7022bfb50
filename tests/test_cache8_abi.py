"""Accumulated attention weights and the 8-bit cache: bad arguments are refused on the host, before anything is
enqueued (no GPU needed), and calls without work return at once."""
import ctypes
import math

import pytest

from paper_2608_27128_amd import binding
from test_cache_ops_abi import BAD_CACHES, E_ARG, E_NULL, E_UNSUP, E_WS, FAKE, I63, arr, struct


def mass(q=FAKE, k=FAKE, dtype=0, d=128, H=2, G=4, cq=(0, 10), ck=(0, 100), qs=(1280, 128), ks=(12800, 128), window=50,
         n_sink=4, scale=0.1, lse=FAKE, old=None, out=FAKE, ws=FAKE, wsb=1 << 40):
    n = 1 if cq is None else len(cq) - 1
    return binding.lib().twinkv_attention_mass(q, k, dtype, d, H, G, n, arr(cq), arr(ck), *qs, *ks, window, n_sink, scale,
                                               lse, old, out, ws, wsb, None)


def test_attention_mass_refusals():
    for name in ("q", "k"):
        assert mass(**{name: None}) == E_NULL, name
        assert mass(**{name: FAKE + 2}) == E_ARG, name
    assert mass(lse=None) == mass(out=None) == mass(cq=None) == mass(ck=None) == E_NULL
    assert mass(d=32) == mass(dtype=-1) == E_UNSUP
    assert mass(H=0) == mass(H=65536) == mass(G=0) == mass(G=1 << 30) == E_ARG
    assert mass(cq=(0, 10, 5), ck=(0, 1, 2)) == mass(cq=(1, 10)) == mass(ck=(0, 1 << 31)) == E_ARG
    assert mass(window=-1) == mass(n_sink=-1) == mass(scale=math.inf) == mass(scale=math.nan) == E_ARG
    assert mass(ks=(12800, 64)) == mass(qs=(-8, 128)) == mass(ks=(12800, 132)) == E_ARG
    assert mass(ck=(0, 0), k=None, out=None) == 0                       # no keys: nothing to write
    prompt = dict(cq=(0, 8192), ck=(0, 8192), window=8192, n_sink=0)
    assert mass(**prompt, ws=None) == mass(**prompt, wsb=100) == E_WS


def test_mass_workspace():
    f = binding.lib().twinkv_mass_workspace_bytes

    def need(cq, ck, H=8, G=4, d=128, window=I63, n_sink=0, dtype=0):
        return f(dtype, d, H, G, len(cq) - 1, arr(cq), arr(ck), window, n_sink)
    assert need((0, 1), (0, 4096)) == 0                                 # few rows: nothing split
    assert need((0, 8192), (0, 8192)) > 0
    assert need((0, 8192), (0, 8192), window=128) < need((0, 8192), (0, 8192))
    assert need(tuple(range(1001)), tuple(range(1001))) > 0             # words of many sequences
    assert need((0, 1), (0, 10), d=96) == -E_UNSUP
    assert need((0, 1), (0, 10), H=0) == need((0, 1), (0, 10), window=-1) == -E_ARG
    assert f(0, 128, 8, 4, 1, None, arr((0, 1)), 1, 0) == -E_NULL


def handle(c):
    return ctypes.addressof(c) if c is not None else None


def compact(c=struct, keys=FAKE, values=FAKE, dtype=0, cu=(0, 100), s=(12800, 128), ret=FAKE, tm=None, pos=FAKE, mo=None,
            n=FAKE, st=FAKE, ws=None, wsb=0):
    c = c() if callable(c) else c
    return binding.lib().twinkv_cache8_compact(keys, values, dtype, arr(cu), *s, *s, ret, handle(c), tm, pos, mo, n, st, ws,
                                               wsb, None)


def append(c=struct, keys=FAKE, values=FAKE, dtype=0, cu=(0, 1), s=(128, 128), n_in=FAKE, n=FAKE, st=FAKE, ws=None, wsb=0):
    c = c() if callable(c) else c
    return binding.lib().twinkv_cache8_append(keys, values, dtype, arr(cu), *s, *s, handle(c), n_in, n, st, ws, wsb, None)


def read(c=struct, n=FAKE, first=None, dtype=0, cu=(0, 64), ko=FAKE, vo=FAKE, ws=None, wsb=0):
    c = c() if callable(c) else c
    return binding.lib().twinkv_cache8_read(handle(c), n, first, dtype, arr(cu), ko, vo, ws, wsb, None)


def attend(c=struct, q=FAKE, dtype=0, G=4, cu=(0, 1), s=(128, 128), n=FAKE, scale=0.1, out=FAKE, os=(128, 128), mi=None,
           mo=None, ws=FAKE, wsb=1 << 40):
    c = c() if callable(c) else c
    return binding.lib().twinkv_cache8_attention(q, dtype, G, arr(cu), *s, handle(c), n, scale, out, *os, None, mi, mo, ws,
                                                 wsb, None)


@pytest.mark.parametrize("call", [compact, append, read, attend])
def test_cache8_refuses_bad_caches(call):
    assert call(None) == E_NULL
    for kw, code in BAD_CACHES:
        assert call(struct(**kw)) == code, kw
    assert call(dtype=9) == E_UNSUP
    assert call(cu=None) == E_NULL
    assert call(cu=(0, -1)) == E_ARG
    many = struct(rows=tuple(32 * i for i in range(1001)))
    assert call(many, cu=tuple(range(1001)), ws=None, wsb=0) == E_WS


def test_cache8_refusals():
    assert compact(keys=None) == compact(values=None) == compact(ret=None) == E_NULL
    assert compact(pos=None) == compact(n=None) == compact(st=None) == compact(tm=FAKE) == E_NULL
    assert compact(keys=FAKE + 8) == compact(s=(12800, 120)) == E_ARG
    assert append(keys=None) == append(n_in=None) == append(n=None) == append(st=None) == E_NULL
    assert append(s=(128, 64)) == E_ARG
    assert read(n=None) == E_NULL
    assert read(ko=FAKE + 4) == E_ARG
    assert attend(q=None) == attend(out=None) == attend(n=None) == attend(mi=FAKE) == E_NULL
    assert attend(G=0) == attend(scale=math.nan) == attend(mi=FAKE + 4, mo=FAKE) == attend(mo=FAKE + 8) == E_ARG
    assert attend(os=(8, 128)) == E_ARG
    assert attend(cu=(0, 0), q=None, out=None) == 0
    big = struct(rows=(0, 1 << 17))
    assert attend(big, ws=None) == attend(big, wsb=64) == attend(big, mo=FAKE, wsb=64) == E_WS
    f = binding.lib().twinkv_cache8_workspace_bytes
    assert f(0) == -E_ARG and f(1) == 0 and f(5000) > 4 * 5000


def test_cache8_attention_workspace():
    f = binding.lib().twinkv_cache8_attention_workspace_bytes

    def need(cq, rows, want, H=8, G=4, d=128, dtype=0):
        return f(dtype, d, H, G, len(cq) - 1, arr(cq), arr(rows), want)
    assert need((0, 1), (0, 512), 0) == need((0, 1), (0, 512), 1) == 0   # one item a head: scores stay in LDS
    long = need((0, 1), (0, 1 << 17), 0)
    assert 0 < long < need((0, 1), (0, 1 << 17), 1)
    assert need((0, 64), (0, 512), 1) > 0                                # more rows than a tile: log-sum-exps
    assert need((0, 1), (0, 512), 0, d=32) == -E_UNSUP
    assert need((0, 1), (0, 512), 0, G=0) == -E_ARG
    assert f(0, 128, 8, 4, 1, arr((0, 1)), None, 0) == -E_NULL


def evict(a=struct, n=FAKE, m=FAKE, pos=None, budget=(10,), sink=4, recent=4, b=None, no=FAKE, mo=None, po=FAKE, ws=None,
          wsb=0):
    a = a() if callable(a) else a
    b = other() if b is None else b
    return binding.lib().twinkv_cache8_evict(handle(a), n, m, pos, arr(budget), sink, recent, handle(b), no, mo, po, ws, wsb,
                                             None)


def other(**kw):
    return struct(**{**dict(k=FAKE + 4096, ks=FAKE + 8192, v=FAKE + 12288, vs=FAKE + 16384), **kw})


def test_evict_refusals():
    for kw, code in BAD_CACHES:
        assert evict(struct(**kw)) == code, kw
    for kw, code in BAD_CACHES:
        assert evict(b=other(**kw)) == code, kw
    assert evict(None) == E_NULL
    assert evict(n=None) == evict(m=None) == evict(no=None) == evict(po=None) == evict(budget=None) == E_NULL
    assert evict(b=other(d=64)) == evict(b=other(H=3)) == evict(b=other(rows=(0, 32, 64))) == E_ARG
    assert evict(budget=(-1,)) == evict(budget=(65,)) == evict(sink=-1) == evict(recent=-1) == E_ARG
    assert evict(m=FAKE + 4) == E_ARG
    assert evict(b=other(v=FAKE)) == evict(b=struct()) == E_ARG          # arrays in common
    rows = tuple(32 * i for i in range(1001))
    assert evict(struct(rows=rows), b=other(rows=rows), budget=(1,) * 1000) == E_WS


def test_binding_refusals():
    import torch
    x = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    z = torch.zeros((2, 8))
    for call in (lambda: binding.attention_mass(x, x, z, 8), lambda: binding.attention_mass(x.half(), x, z, 8),
                 lambda: binding.Cache8.empty(2, [30], 128, device="cpu"),
                 lambda: binding.Cache8(*(torch.zeros((1, 1, 1)),) * 4, [0, 33]),
                 lambda: binding.Cache8(*(torch.zeros((1, 32, 64)),) * 4, [0, 32])):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_inputs_that_require_a_gradient():
    """Before anything else, so that CPU tensors show it."""
    import torch
    x = torch.zeros((2, 8, 128), dtype=torch.bfloat16, requires_grad=True)
    z = torch.zeros((2, 8))
    with pytest.raises(ValueError, match="no gradient"):
        binding.attention_mass(x, x, z, 8)
    with pytest.raises(ValueError, match="no gradient"):
        binding.attention_mass(x.detach(), x.detach(), z.requires_grad_(), 8)
    with pytest.raises(ValueError, match="no gradient"):
        binding.cache8_attention(x, None, None)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        binding.attention_mass(x, x, z, 8)
