"""The operators around the cache refuse bad arguments on the host, before anything is enqueued (no GPU
needed), and calls without work return at once."""
import ctypes
import math

import pytest

from paper_2608_27128_amd import binding

E_NULL, E_ARG, E_UNSUP, E_WS = 1, 2, 3, 4
FAKE = 0x100000  # 16-byte aligned stand-in for a device pointer; never dereferenced
I63 = (1 << 63) - 1


def arr(v):
    return None if v is None else (ctypes.c_int64 * len(v))(*v)


def rope(q=FAKE, k=FAKE, dtype=0, d=128, hq=4, hk=1, T=8, qs=(128, 512), ks=(1024, 128), qw=FAKE, kw=None, eps=1e-6,
         table=FAKE, n_pos=10, pos=FAKE, qo=FAKE, qos=(1024, 128), ko=FAKE, kos=(1024, 128)):
    return binding.lib().twinkv_qk_norm_rope(q, k, dtype, d, hq, hk, T, *qs, *ks, qw, kw, eps, table, n_pos, pos, qo,
                                             *qos, ko, *kos, None)


def test_norm_rope_refusals():
    assert rope(q=None) == E_NULL
    assert rope(k=None) == E_NULL
    assert rope(qo=None) == E_NULL
    assert rope(ko=None) == E_NULL
    assert rope(pos=None) == E_NULL
    assert rope(d=96) == E_UNSUP
    assert rope(dtype=2) == E_UNSUP
    assert rope(hq=-1) == E_ARG
    assert rope(hq=60000, hk=60000) == E_ARG
    assert rope(T=-1) == E_ARG
    assert rope(T=1 << 31) == E_ARG
    assert rope(eps=-1.0) == E_ARG
    assert rope(eps=math.nan) == E_ARG
    assert rope(n_pos=-1) == E_ARG
    assert rope(q=FAKE + 8) == E_ARG
    assert rope(qw=FAKE + 4) == E_ARG
    assert rope(table=FAKE + 8) == E_ARG
    assert rope(qs=(128, 100)) == E_ARG       # tokens overlap
    assert rope(qs=(128, 516)) == E_ARG       # not a multiple of 16 bytes
    assert rope(kos=(-128, 128)) == E_ARG
    assert rope(T=0, q=None, k=None, qo=None, ko=None, pos=None) == 0
    assert rope(hq=0, hk=0, q=None, k=None, qo=None, ko=None) == 0


def sink(q=FAKE, k=FAKE, v=FAKE, dtype=0, d=128, H=2, G=4, cq=(0, 10), ck=(0, 100), qs=(1280, 128), ks=(12800, 128),
         window=50, n_sink=4, scale=0.1, out=FAKE, os=(1280, 128), lse=None, ws=FAKE, wsb=1 << 40):
    n = 1 if cq is None else len(cq) - 1
    return binding.lib().twinkv_sink_attention(q, k, v, dtype, d, H, G, n, arr(cq), arr(ck), *qs, *ks, *ks, window,
                                               n_sink, scale, out, *os, lse, ws, wsb, None)


def test_sink_attention_refusals():
    for name in ("q", "k", "v", "out"):
        assert sink(**{name: None}) == E_NULL, name
        assert sink(**{name: FAKE + 2}) == E_ARG, name
    assert sink(cq=None) == E_NULL
    assert sink(ck=None) == E_NULL
    assert sink(d=32) == E_UNSUP
    assert sink(dtype=-1) == E_UNSUP
    assert sink(H=0) == E_ARG
    assert sink(H=65536) == E_ARG
    assert sink(G=0) == E_ARG
    assert sink(G=1 << 30) == E_ARG
    assert sink(cq=(0, 10, 5), ck=(0, 1, 2)) == E_ARG
    assert sink(cq=(1, 10)) == E_ARG
    assert sink(ck=(0, 1 << 31)) == E_ARG
    assert sink(window=-1) == E_ARG
    assert sink(n_sink=-1) == E_ARG
    assert sink(scale=math.inf) == E_ARG
    assert sink(ks=(12800, 64)) == E_ARG
    assert sink(cq=(0, 0), q=None, out=None) == 0           # no queries


def test_attention_workspace():
    f = binding.lib().twinkv_attention_workspace_bytes

    def need(cq, ck, H=8, G=4, d=128, window=I63, n_sink=0, dtype=0):
        return f(dtype, d, H, G, len(cq) - 1, arr(cq), arr(ck), window, n_sink)
    assert need((0, 1), (0, 128)) == 0                       # one short sequence: nothing split
    long = need((0, 1), (0, 131072))
    assert long > 0 and need((0, 1), (0, 131072), window=256) < long
    assert need(tuple(range(1001)), tuple(range(1001))) > 0  # words of many sequences
    assert need((0, 131072), (0, 131072)) == 0               # a whole prompt fills the machine unsplit
    assert sink(cq=(0, 1), ck=(0, 131072), window=1 << 20, ws=None) == E_WS
    assert sink(cq=(0, 1), ck=(0, 131072), window=1 << 20, wsb=100) == E_WS
    assert need((0, 1), (0, 10), d=96) == -E_UNSUP
    assert need((0, 1), (0, 10), H=0) == -E_ARG
    assert need((0, 1), (0, 10), window=-1) == -E_ARG
    assert f(0, 128, 8, 4, 1, None, arr((0, 1)), 1, 0) == -E_NULL


def struct(d=128, H=2, rows=(0, 64), k=FAKE, ks=FAKE, v=FAKE, vs=FAKE, n=None):
    cu = arr(rows)
    s = binding._Cache4Struct(d, H, len(rows) - 1 if n is None else n, ctypes.cast(cu, binding._PI64), k, ks, v, vs)
    s.keep = cu
    return s


BAD_CACHES = [(dict(d=96), E_UNSUP), (dict(H=0), E_ARG), (dict(H=70000), E_ARG), (dict(rows=(0, 40)), E_ARG),
              (dict(rows=(32, 64)), E_ARG), (dict(rows=(0, 64, 32)), E_ARG), (dict(n=0), E_ARG), (dict(k=None), E_NULL),
              (dict(ks=None), E_NULL), (dict(v=None), E_NULL), (dict(vs=None), E_NULL), (dict(k=FAKE + 4), E_ARG),
              (dict(vs=FAKE + 1), E_ARG)]


def compact(c=None, keys=FAKE, values=FAKE, dtype=0, cu=(0, 100), s=(12800, 128), ret=FAKE, pos=FAKE, n=FAKE, st=FAKE,
            ws=None, wsb=0, handle=True):
    c = c or struct()
    return binding.lib().twinkv_cache4_compact(keys, values, dtype, arr(cu), *s, *s, ret,
                                               ctypes.addressof(c) if handle else None, pos, n, st, ws, wsb, None)


def append(c=None, keys=FAKE, values=FAKE, dtype=0, cu=(0, 1), s=(128, 128), n_in=FAKE, n=FAKE, st=FAKE, ws=None, wsb=0,
           handle=True):
    c = c or struct()
    return binding.lib().twinkv_cache4_append(keys, values, dtype, arr(cu), *s, *s,
                                              ctypes.addressof(c) if handle else None, n_in, n, st, ws, wsb, None)


def read(c=None, n=FAKE, first=None, dtype=0, cu=(0, 64), ko=FAKE, vo=FAKE, ws=None, wsb=0, handle=True):
    c = c or struct()
    return binding.lib().twinkv_cache4_read(ctypes.addressof(c) if handle else None, n, first, dtype, arr(cu), ko, vo, ws,
                                            wsb, None)


def attend(c=None, q=FAKE, dtype=0, G=4, cu=(0, 1), s=(128, 128), n=FAKE, scale=0.1, out=FAKE, os=(128, 128), ws=FAKE,
           wsb=1 << 40, handle=True):
    c = c or struct()
    return binding.lib().twinkv_cache4_attention(q, dtype, G, arr(cu), *s, ctypes.addressof(c) if handle else None, n,
                                                 scale, out, *os, None, ws, wsb, None)


@pytest.mark.parametrize("call", [compact, append, read, attend])
def test_cache4_refuses_bad_caches(call):
    assert call(handle=False) == E_NULL
    for kw, code in BAD_CACHES:
        assert call(struct(**kw)) == code, kw
    assert call(dtype=9) == E_UNSUP
    assert call(cu=None) == E_NULL
    assert call(cu=(0, -1)) == E_ARG
    many = struct(rows=tuple(32 * i for i in range(1001)))
    assert call(many, cu=tuple(range(1001)), ws=None, wsb=0) == E_WS


def test_cache4_refusals():
    assert compact(keys=None) == compact(values=None) == compact(ret=None) == E_NULL
    assert compact(pos=None) == compact(n=None) == compact(st=None) == E_NULL
    assert compact(keys=FAKE + 8) == E_ARG
    assert compact(s=(12800, 120)) == E_ARG
    assert append(keys=None) == append(n_in=None) == append(n=None) == append(st=None) == E_NULL
    assert append(s=(128, 64)) == E_ARG
    assert read(n=None) == E_NULL
    assert read(ko=FAKE + 4) == E_ARG
    assert attend(q=None) == attend(out=None) == attend(n=None) == E_NULL
    assert attend(G=0) == E_ARG
    assert attend(scale=math.nan) == E_ARG
    assert attend(cu=(0, 0), q=None, out=None) == 0
    big = struct(rows=(0, 1 << 17))
    assert attend(big, ws=None) == attend(big, wsb=64) == E_WS
    assert binding.lib().twinkv_cache4_workspace_bytes(0) == -E_ARG
    assert binding.lib().twinkv_cache4_workspace_bytes(1) == 0
    assert binding.lib().twinkv_cache4_workspace_bytes(5000) > 4 * 5000


def test_binding_refusals():
    import torch
    x = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    for call in (lambda: binding.qk_norm_rope(None, None), lambda: binding.qk_norm_rope(x, x),
                 lambda: binding.qk_norm_rope(x.half(), None), lambda: binding.qk_norm_rope(x[0, 0], None),
                 lambda: binding.sink_attention(x, x, x, 8), lambda: binding.sink_attention(x.half(), x, x, 8),
                 lambda: binding.Cache4.empty(2, [30], 128, device="cpu"),
                 lambda: binding.Cache4(*(torch.zeros((1, 1, 1)),) * 4, [0, 33])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("stride", [0, 8, 120])
def test_heads_of_an_output_may_not_overlap(stride):
    assert rope(qos=(stride, 128)) == E_ARG
    assert rope(hk=2, kos=(stride, 128)) == E_ARG
    assert sink(os=(stride, 128)) == E_ARG
    assert attend(os=(stride, 128)) == E_ARG
    assert rope(T=0, q=None, k=None, qo=None, ko=None, pos=None, qos=(stride, 128)) == 0
