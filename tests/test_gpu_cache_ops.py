"""The operators around the cache on the GPU against plain 64-bit forms (cache_ops_ref.py): norm and
rotation, attention over a window and sinks, the 4-bit cache and the attention over it.  Tolerances are
those that the number formats give (attention_bounds); the 4-bit values are exact."""
import math

import numpy as np
import pytest

import cache_ops_ref as ref
from paper_2608_27128_amd import binding

pytestmark = pytest.mark.gpu
OK, MISMATCH, NONFINITE = 0, 1, 2


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype="bf16"):
    import torch
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def table(n, d, theta=1e4):
    import torch
    f = theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int64)


# ---------------------------------------------------------------- norm and rotation

def rope_tol(want, d, bf16):
    # the mean of d squares (d roundings, halved by the root) and a few more, of the row's largest element
    top = want.abs().amax(-1, keepdim=True).nan_to_num()
    tol = (d / 2 + 12) * ref.U * top * 1.5
    return tol + (1.01 * ref.U16 * want.abs().nan_to_num() if bf16 else 0.0)


def check_rope(got, want, d, dtype):
    import torch
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    err = (got.double() - want).abs().nan_to_num()
    assert bool((err <= rope_tol(want, d, dtype == "bf16")).all()), float(err.max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,hq,hk,major", [(1, 4, 1, True), (3, 5, 2, False), (65, 32, 8, True), (33, 0, 3, True),
                                           (17, 9, 0, False), (1000, 12, 3, True), (700, 70, 9, False)])
def test_norm_rope(T, hq, hk, major, dtype, d):
    import torch
    g = gen(T * 7 + d)

    def rows(h):
        x = randn(g, T, h, d, dtype=dtype).transpose(0, 1)
        return None if h == 0 else (x if major else x.contiguous())
    q, k = rows(hq), rows(hk)
    qw, kw = 1 + 0.3 * randn(g, d, dtype="f32"), 1 + 0.3 * randn(g, d, dtype="f32")
    rope = table(50, d)
    pos = torch.randint(0, 50, (T,), generator=g, device="cuda", dtype=torch.int32)
    for wq, wk, r in ((qw, kw, rope), (None, kw, rope), (qw, None, rope), (qw, kw, None)):
        out = binding.qk_norm_rope(q, k, wq, wk, 1e-5, r, pos)
        for name, x, w in (("q", q, wq), ("k", k, wk)):
            if x is not None:
                check_rope(out[name], ref.norm_rope(x.double(), w, 1e-5, r, pos), d, dtype)


def test_norm_rope_in_place_and_outside_the_table():
    import torch
    g = gen(1)
    d, T = 128, 300
    q, k = randn(g, T, 12, d).transpose(0, 1), randn(g, 2, T, d)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) - 1
    pos[7] = 1 << 30
    rope = table(200, d)
    w = torch.ones(d, device="cuda")
    want = binding.qk_norm_rope(q, k, w, w, 0.0, rope, pos)
    check_rope(want["k"], ref.norm_rope(k.double(), w, 0.0, rope, pos), d, "bf16")
    bad = torch.isnan(want["q"]).all(-1).all(0)
    assert bad.nonzero().squeeze(1).tolist() == [0, 7] + list(range(201, 300))
    binding.qk_norm_rope(q, k, w, w, 0.0, rope, pos, q_out=q, k_out=k)
    for a, b in ((q, want["q"]), (k, want["k"])):
        assert torch.equal(a.contiguous().view(torch.int16), b.view(torch.int16))


def test_norm_rope_zero_rows_and_no_tokens():
    import torch
    z = torch.zeros((2, 5, 64), device="cuda")
    out = binding.qk_norm_rope(z, None, torch.ones(64, device="cuda"), None, 1e-6)
    assert torch.equal(out["q"], z)
    empty = torch.zeros((2, 0, 64), device="cuda")
    assert binding.qk_norm_rope(empty, empty)["k"].shape == (2, 0, 64)


# ---------------------------------------------------------------- attention over a window and sinks

def check_attention(got, q, k, v, cu_q, cu_k, seen_of, scale, dtype, lse=None, heads=None):
    """Every head (or those listed) of every sequence against the 64-bit form."""
    Hq, _, d = q.shape
    G = Hq // k.shape[0]
    for s in range(len(cu_q) - 1):
        a, b = int(cu_q[s]), int(cu_q[s + 1])
        x, y = int(cu_k[s]), int(cu_k[s + 1])
        for h in heads if heads is not None else range(Hq):
            seen = seen_of(s, h, b - a, y - x).to(q.device)
            o, e, mass, size = ref.softmax_rows(q[h, a:b].double(), k[h // G, x:y].double(), v[h // G, x:y].double(),
                                                seen, scale)
            tol, tol_e = ref.attention_bounds(o, e, mass, size, y - x, d, dtype == "bf16")
            err = (got[h, a:b].double() - o).abs()
            assert bool((err <= tol).all()), (s, h, float((err - tol).max()))
            if lse is not None:
                none = e == -math.inf
                assert bool((lse[h, a:b][none] == -math.inf).all())
                assert bool(((lse[h, a:b].double() - e).abs()[~none] <= tol_e[~none]).all()), (s, h)


ATTN = [  # lens, queries (0: all), window, sinks, group
    ((1,), (0,), 1, 0, 1), ((5,), (0,), 3, 1, 4), ((33,), (0,), 1000, 0, 3), ((70,), (0,), 16, 4, 4),
    ((200,), (0,), 31, 33, 2), ((300,), (1,), 64, 4, 4), ((300,), (1,), 1 << 40, 0, 16), ((513,), (7,), 100, 2, 5),
    ((257,), (0,), 0, 0, 2), ((130,), (0,), 0, 5, 2), ((90, 1, 0, 400, 64), (3, 0, 0, 1, 64), 50, 4, 4),
    ((40, 10), (50, 10), 20, 2, 2), ((1500,), (129,), 300, 40, 4), ((260,), (256,), 1 << 20, 0, 1),
    ((640,), (0,), 128, 64, 8), ((2100,), (2,), 1 << 20, 0, 20)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_sink_attention(case, dtype, d):
    lens, nq, window, sink, G = ATTN[case]
    nq = [m if m else (n if len(lens) == 1 else 0) for m, n in zip(nq, lens)]
    g = gen(100 + case)
    H = 2
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, H * G, sum(nq), d, dtype=dtype)
    k, v = randn(g, H, sum(lens), d, dtype=dtype), randn(g, H, sum(lens), d, dtype=dtype)
    k = k + 2 * randn(g, H, 1, d, dtype=dtype)
    got = binding.sink_attention(q, k, v, window, sink, None, cu_q, cu_k, want_lse=True)
    check_attention(got["out"], q, k, v, cu_q, cu_k, lambda s, h, m, n: ref.seen_by(m, n, window, sink), d ** -0.5,
                    dtype, got["lse"], heads=sorted({0, G - 1, H * G - 1}))


def test_sink_attention_token_major_strides_and_out():
    import torch
    g = gen(3)
    T, H, G, d = 333, 2, 4, 128
    qkv = randn(g, T, H * G + 2 * H, d)
    q, k, v = (x.transpose(0, 1) for x in qkv.split([H * G, H, H], 1))
    out = torch.zeros((T, H * G, d), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    binding.sink_attention(q, k, v, 100, 4, 0.1, out=out)
    want = binding.sink_attention(q.contiguous(), k.contiguous(), v.contiguous(), 100, 4, 0.1)["out"]
    assert torch.equal(out, want)
    check_attention(out, q, k, v, [0, T], [0, T], lambda s, h, m, n: ref.seen_by(m, n, 100, 4), 0.1, "bf16", heads=[5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m", [(150, 150), (700, 700), (500, 1), (900, 40)])
def test_sink_attention_unseen_values_do_not_matter(n, m, dtype):
    """NaN and infinities in keys and values reach exactly the queries that see them."""
    import torch
    g = gen(n + m)
    H, G, d, W, sink = 2, 4, 128, 40, 3
    q = randn(g, H * G, m, d, dtype=dtype)
    k, v = randn(g, H, n, d, dtype=dtype), randn(g, H, n, d, dtype=dtype)
    clean = binding.sink_attention(q, k, v, W, sink, None, [0, m], [0, n], want_lse=True)
    seen = ref.seen_by(m, n, W, sink).cuda()
    for j, what in ((1, math.nan), (n // 3, math.inf), (n - 20, math.nan), (n - 1, -math.inf), (n // 2, math.nan)):
        k2, v2 = k.clone(), v.clone()
        v2[:, j, 5] = what
        got = binding.sink_attention(q, k2, v2, W, sink, None, [0, m], [0, n])["out"]
        hit = torch.zeros((H * G, m, d), dtype=torch.bool, device="cuda")
        hit[:, seen[:, j], 5] = True
        assert torch.equal(got[~hit], clean["out"][~hit]), (j, what)
        assert not bool(torch.isfinite(got[hit]).any()), (j, what)
        k2[:, j] = what if math.isnan(what) else math.nan
        got = binding.sink_attention(q, k2, v, W, sink, None, [0, m], [0, n], want_lse=True)
        rows = seen[:, j]
        assert torch.equal(got["out"][:, ~rows], clean["out"][:, ~rows])
        assert torch.equal(got["lse"][:, ~rows], clean["lse"][:, ~rows])
        assert bool(torch.isnan(got["out"][:, rows]).all())


def test_sink_attention_large_scores():
    """Scores of thousands: the maximum moves many times, and nothing overflows."""
    g = gen(9)
    d, n = 64, 900
    q, k, v = 30 * randn(g, 1, 3, d, dtype="f32"), randn(g, 1, n, d, dtype="f32"), randn(g, 1, n, d, dtype="f32")
    import torch
    k = k * torch.linspace(0.0, 3.0, n, device="cuda")[None, :, None]
    got = binding.sink_attention(q, k, v, n, 0, 1.0, [0, 3], [0, n], want_lse=True)
    check_attention(got["out"], q, k, v, [0, 3], [0, n], lambda s, h, m, nk: ref.seen_by(m, nk, n, 0), 1.0, "f32", got["lse"])


def test_sink_attention_many_sequences():
    """More sequences than the kernel arguments hold: the words go through the workspace."""
    g = gen(17)
    S, H, G, d = 400, 1, 2, 64
    lens = [(i * 37) % 50 for i in range(S)]
    nq = [min(n, 1 + i % 3) for i, n in enumerate(lens)]
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, H * G, int(cu_q[-1]), d)
    k, v = randn(g, H, int(cu_k[-1]), d), randn(g, H, int(cu_k[-1]), d)
    got = binding.sink_attention(q, k, v, 20, 2, None, cu_q, cu_k, want_lse=True)
    check_attention(got["out"], q, k, v, cu_q, cu_k, lambda s, h, m, n: ref.seen_by(m, n, 20, 2), d ** -0.5, "bf16", got["lse"])


# ---------------------------------------------------------------- the 4-bit cache

def compact_ref(keys, retained, cu, s, h):
    a, b = int(cu[s]), int(cu[s + 1])
    pos = retained[h, a:b].nonzero().squeeze(1)
    return pos, ref.quantise(keys[h, a + pos].double())[0]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,spare", [((100,), 0), ((1, 0, 33, 515), 40), ((20011,), 7)])
def test_cache4_compact(lens, spare, dtype, d):
    import torch
    g = gen(sum(lens) + d)
    H, T, cu = 3, sum(lens), cum(lens)
    keys = randn(g, T, H, d, dtype=dtype).transpose(0, 1) * 3
    values = randn(g, H, T, d, dtype=dtype)
    keys[0, :, :8] *= 1e-3
    values[1, ::3] *= 1e4
    values[2, ::5] = 0
    ret = (torch.rand((H, T), generator=g, device="cuda") < 0.4).to(torch.uint8) * 7  # any nonzero byte keeps
    caps = [int(ret[:, a:b].ne(0).sum(1).max()) + spare if b > a else 0 for a, b in zip(cu[:-1], cu[1:])]
    cache = binding.Cache4.empty(H, caps, d)
    for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        x.fill_(255)
    got = binding.cache4_compact(keys, values, ret, cache, cu)
    assert bool((got["status"] == OK).all())
    kv = binding.cache4_read(cache, got["len"], keys.dtype)
    for s in range(len(lens)):
        r0, r1 = int(cache.cu_rows[s]), int(cache.cu_rows[s + 1])
        for h in range(H):
            pos, want = compact_ref(keys, ret, cu, s, h)
            n = len(pos)
            assert int(got["len"][h, s]) == n
            assert torch.equal(got["pos"][h, r0:r0 + n].long(), pos)
            assert bool((got["pos"][h, r0 + n:r1] == -1).all())
            _, want_v = compact_ref(values, ret, cu, s, h)
            assert torch.equal(kv["keys"][h, r0:r0 + n].double(), want)
            assert torch.equal(kv["values"][h, r0:r0 + n].double(), want_v)
            assert not bool(kv["keys"][h, r0 + n:r1].any()) and not bool(kv["values"][h, r0 + n:r1].any())


def test_cache4_every_bf16():
    """Every bf16 number, alone in its group and beside a larger one, has the value the format gives it."""
    import torch
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16)
    rows = torch.zeros((1, 65536, 64), dtype=torch.bfloat16, device="cuda")
    rows[0, :, 0] = x                          # alone
    rows[0, :, 32] = x
    rows[0, :, 33] = 5.0 * x                   # inside a group's range
    cache = binding.Cache4.empty(1, 65536, 64)
    ones = torch.ones((1, 65536), dtype=torch.uint8, device="cuda")
    got = binding.cache4_compact(rows, rows, ones, cache)
    assert int(got["status"]) == NONFINITE
    kv = binding.cache4_read(cache, got["len"], torch.float32)
    want, _ = ref.quantise(rows[0].double())
    assert torch.equal(kv["keys"][0].double(), want)
    assert torch.equal(kv["values"][0].double(), want)


def test_cache4_states():
    """A problem that keeps more than its rows stores nothing; a non-finite group is zeros and reported;
    the other problems are as without them."""
    import torch
    g = gen(5)
    H, d, lens = 2, 128, (100, 60)
    cu, T = cum(lens), 160
    keys, values = randn(g, H, T, d), randn(g, H, T, d)
    ret = torch.ones((H, T), dtype=torch.uint8, device="cuda")
    ret[0, 40:100] = 0
    keys[0, 120, 70] = math.inf
    values[0, 121, 3] = math.nan
    cache = binding.Cache4.empty(H, [64, 64], d)
    got = binding.cache4_compact(keys, values, ret, cache, cu)
    assert got["len"].tolist() == [[40, 60], [0, 60]]
    assert got["status"].tolist() == [[OK, NONFINITE], [MISMATCH, OK]]
    assert bool((got["pos"][1, :64] == -1).all())
    kv = binding.cache4_read(cache, got["len"], torch.bfloat16)
    for h, s in ((0, 0), (0, 1), (1, 1)):
        n, r0, a = int(got["len"][h, s]), int(cache.cu_rows[s]), int(cu[s])
        for x, y in ((keys, kv["keys"]), (values, kv["values"])):
            assert torch.equal(y[h, r0:r0 + n].double(), ref.quantise(x[h, a:a + n].double())[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache4_append(dtype, d):
    """Appending in steps of any size gives what appending all at once gives, and touches nothing else."""
    import torch
    g = gen(d)
    H, caps = 3, [96, 320, 32]
    steps = [[3, 0, 1], [1, 1, 1], [8, 130, 5], [0, 1, 24], [13, 150, 0], [40, 7, 1]]
    cache = binding.Cache4.empty(H, caps, d)
    length = torch.tensor([[0, 0, 0], [5, 1, 0], [20, 30, 7]], dtype=torch.int32, device="cuda")
    rows = {n: torch.zeros((H, sum(caps), d), dtype=torch.float64, device="cuda") for n in ("keys", "values")}
    start = length.clone()
    have = length.tolist()
    zero = randn(g, H, 0, d, dtype=dtype)
    assert binding.cache4_append(zero, zero, cache, length, [0, 0, 0, 0])["len"].tolist() == have
    for k, n in enumerate(steps):
        cu = cum(n)
        keys, values = randn(g, int(cu[-1]), H, d, dtype=dtype).transpose(0, 1), randn(g, H, int(cu[-1]), d, dtype=dtype)
        got = binding.cache4_append(keys, values, cache, length, cu, len_out=length if k % 2 else None)
        length = got["len"]
        for h in range(H):
            for s in range(3):
                fits = have[h][s] + n[s] <= caps[s]
                assert int(got["status"][h, s]) == (OK if fits else MISMATCH)
                if fits:
                    r, a = int(cache.cu_rows[s]) + have[h][s], int(cu[s])
                    rows["keys"][h, r:r + n[s]] = ref.quantise(keys[h, a:a + n[s]].double())[0]
                    rows["values"][h, r:r + n[s]] = ref.quantise(values[h, a:a + n[s]].double())[0]
                    have[h][s] += n[s]
        assert length.tolist() == have
        first = start
        kv = binding.cache4_read(cache, length, keys.dtype)
        for h in range(H):
            for s in range(3):
                a, b = int(cache.cu_rows[s]) + int(first[h, s]), int(cache.cu_rows[s]) + have[h][s]
                for name in ("keys", "values"):
                    assert torch.equal(kv[name][h, a:b].double(), rows[name][h, a:b]), (k, h, s, name)


def test_cache4_append_states():
    import torch
    g = gen(8)
    H, d = 2, 64
    cache = binding.Cache4.empty(H, [32, 64], d)
    keys, values = randn(g, H, 3, d), randn(g, H, 3, d)
    values[1, 2, 40] = math.nan
    length = torch.tensor([[-1, 5], [31, 64]], dtype=torch.int32, device="cuda")
    got = binding.cache4_append(keys, values, cache, length, [0, 1, 3])
    assert got["len"].tolist() == [[-1, 7], [32, 64]]
    assert got["status"].tolist() == [[MISMATCH, OK], [OK, MISMATCH]]
    length = torch.tensor([[0, 0], [0, 62]], dtype=torch.int32, device="cuda")
    got = binding.cache4_append(keys, values, cache, length, [0, 1, 3])
    assert got["status"].tolist() == [[OK, OK], [OK, NONFINITE]]
    kv = binding.cache4_read(cache, got["len"], torch.float32)
    want = ref.quantise(values[1, 2].double())[0]
    assert not bool(want[32:].any()) and torch.equal(kv["values"][1, 32 + 63].double(), want)
    # many at once: lengths and states come before the rows there
    many = randn(g, H, 200, d)
    many[0, 190, 0] = math.inf
    big = binding.Cache4.empty(H, [256, 32], d)
    length = torch.tensor([[56, 3], [57, 4]], dtype=torch.int32, device="cuda")
    got = binding.cache4_append(many, many, big, length, [0, 200, 200], len_out=length)
    assert got["len"].tolist() == [[256, 3], [57, 4]]
    assert got["status"].tolist() == [[NONFINITE, OK], [MISMATCH, OK]]


def test_cache4_read_ranges():
    import torch
    g = gen(11)
    H, d, S = 2, 128, 3
    cache = binding.Cache4.empty(H, [64, 96, 32], d)
    keys = randn(g, H, 192, d)
    ones = torch.ones((H, 192), dtype=torch.uint8, device="cuda")
    length = binding.cache4_compact(keys, keys, ones, cache, cache.cu_rows)["len"] - 9
    whole = binding.cache4_read(cache, length, torch.float32)
    first = torch.tensor([[-3, 50, 31], [60, 7, 1 << 30]], dtype=torch.int32, device="cuda")
    cu = [0, 13, 53, 60]
    got = binding.cache4_read(cache, length, torch.float32, first=first, cu_out=cu)
    only = binding.cache4_read(cache, length, torch.float32, first=first, cu_out=cu, want_keys=False)
    assert "keys" not in only and torch.equal(only["values"], got["values"])
    for h in range(H):
        for s in range(S):
            for r in range(cu[s + 1] - cu[s]):
                row = int(first[h, s]) + r
                for name in ("keys", "values"):
                    x = got[name][h, cu[s] + r]
                    if 0 <= row < int(length[h, s]):
                        assert torch.equal(x, whole[name][h, int(cache.cu_rows[s]) + row])
                    else:
                        assert not bool(x.any())


ATTN4 = [  # capacities, lengths per head, queries per sequence, group
    ((32,), [[1]], (1,), 1), ((32,), [[0]], (2,), 4), ((64,), [[33]], (1,), 4), ((96,), [[90]], (5,), 3),
    ((256, 32, 160), [[256, 31, 100], [200, 0, 129]], (1, 1, 1), 4), ((512,), [[500], [3]], (7,), 4),
    ((640, 64), [[640, 1], [65, 64]], (0, 9), 2), ((4096,), [[4001]], (1,), 16), ((1024,), [[1000]], (33,), 1),
    ((8192,), [[8190]], (2,), 20), ((64000, 4096), [[63000, 4000]] * 8, (5, 3), 10)]


def fill_cache(g, H, caps, d, dtype):
    import torch
    C = int(sum(caps))
    keys = randn(g, H, C, d, dtype=dtype) + 2 * randn(g, H, 1, d, dtype=dtype)
    values = randn(g, H, C, d, dtype=dtype)
    cache = binding.Cache4.empty(H, caps, d)
    ones = torch.ones((H, C), dtype=torch.uint8, device="cuda")
    got = binding.cache4_compact(keys, values, ones, cache, cache.cu_rows)
    return cache, binding.cache4_read(cache, got["len"], torch.float32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTN4)))
def test_cache4_attention(case, dtype, d):
    import torch
    caps, lens, nq, G = ATTN4[case]
    g = gen(200 + case)
    H = len(lens)
    cache, kv = fill_cache(g, H, caps, d, dtype)
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # rows that are not in use may hold anything
    for s, c in enumerate(caps):
        r0 = int(cache.cu_rows[s])
        for h in range(H):
            n = lens[h][s]
            cache.k_codes[h, r0 + n:r0 + c] = 255
            cache.k_scales[h, r0 + n:r0 + c] = 255
            b0 = r0 // 8 + (n + 7) // 8
            cache.v_codes[h, b0:(r0 + c) // 8] = 255
            cache.v_scales[h, b0:(r0 + c) // 8] = 255
            if n % 8:
                cache.v_scales[h, b0 - 1, :, n % 8:] = 255
    cu_q = cum(nq)
    q = randn(g, H * G, int(cu_q[-1]), d, dtype=dtype)
    got = binding.cache4_attention(q, cache, length, 0.11, cu_q, want_lse=True)

    def seen(s, h, m, n):
        at = torch.arange(n)[None, :]
        return at < (lens[h // G][s] - (m - 1 - torch.arange(m)))[:, None]
    check_attention(got["out"], q, kv["keys"], kv["values"], cu_q, cache.cu_rows, seen, 0.11, dtype, got["lse"],
                    heads=sorted({0, G - 1, H * G - 1}))


def test_cache4_many_sequences():
    """More sequences than the kernel arguments hold, through all four calls."""
    import torch
    g = gen(23)
    S, H, d = 300, 2, 64
    lens = [(i * 13) % 40 for i in range(S)]
    cu, T = cum(lens), sum(lens)
    keys, values = randn(g, H, T, d), randn(g, H, T, d)
    ret = torch.ones((H, T), dtype=torch.uint8, device="cuda")
    cache = binding.Cache4.empty(H, [n + 2 for n in lens], d)
    got = binding.cache4_compact(keys, values, ret, cache, cu)
    one = binding.cache4_append(keys[:, :S], values[:, :S], cache, got["len"], np.arange(S + 1))
    kv = binding.cache4_read(cache, one["len"], torch.float32)
    q = randn(g, H * 2, S, d)
    out = binding.cache4_attention(q, cache, one["len"], None, np.arange(S + 1), want_lse=True)
    for s in (0, 1, 100, 298, 299):
        n = lens[s]
        r0 = int(cache.cu_rows[s])
        assert one["len"][:, s].tolist() == [n + 1] * H
        want = torch.cat([keys[:, int(cu[s]):int(cu[s]) + n], keys[:, s:s + 1]], 1).double()
        assert torch.equal(kv["keys"][:, r0:r0 + n + 1].double(), ref.quantise(want)[0])
    check_attention(out["out"], q, kv["keys"], kv["values"], np.arange(S + 1), cache.cu_rows,
                    lambda s, h, m, n: (torch.arange(n)[None, :] < lens[s] + 1).expand(m, n), d ** -0.5, "bf16", out["lse"], heads=[3])


# ---------------------------------------------------------------- streams, graphs, determinism

def test_streams_and_graph():
    """The calls run on the current stream, and a captured decode step replays with new inputs."""
    import torch
    g = gen(31)
    H, G, d, S = 2, 4, 128, 3
    caps = [400, 64, 2016]
    cache, _ = fill_cache(g, H, [(c + 31) // 32 * 32 for c in caps], d, "bf16")
    length = torch.tensor([[390, 5, 2000], [100, 60, 1999]], dtype=torch.int32, device="cuda")
    qw = torch.ones(d, device="cuda")
    rope, pos = table(3000, d), torch.tensor([390, 60, 2000], dtype=torch.int32, device="cuda")
    q, k, v = randn(g, H * G, S, d), randn(g, H, S, d), randn(g, H, S, d)
    cu = np.arange(S + 1)

    def step():
        r = binding.qk_norm_rope(q, k, qw, qw, 1e-6, rope, pos)
        grown = binding.cache4_append(r["k"], v, cache, length, cu)
        return binding.cache4_attention(r["q"], cache, grown["len"], None, cu, want_lse=True)

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = step()
    torch.cuda.current_stream().wait_stream(side)
    for n in ("out", "lse"):
        assert torch.equal(first[n], again[n])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step()
    for t in range(4):
        q.copy_(randn(g, H * G, S, d))
        v.copy_(randn(g, H, S, d))
        graph.replay()
        torch.cuda.synchronize()
        replayed = {n: held[n].clone() for n in held}
        eager = step()
        torch.cuda.synchronize()
        for n in ("out", "lse"):
            assert torch.equal(replayed[n], eager[n]), (t, n)


# shapes that take each of the attention's ways: keys split or not, fp32 waves on row tiles of their own,
# many bf16 rows whole and split, chunks of a prompt over long keys
WAYS = [((700,), (0,), 40, 4, 4, 8), ((2500,), (40,), 1 << 20, 0, 4, 8), ((5000,), (64,), 1 << 20, 4, 2, 8),
        ((9000,), (300,), 3000, 4, 4, 2), ((300,) * 16, (33,) * 16, 1 << 20, 0, 1, 8), ((4200,), (513,), 70, 10, 8, 4),
        ((1300, 40, 3000), (1300, 1, 200), 500, 16, 4, 2)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(WAYS)))
def test_sink_attention_every_way(case, dtype, d):
    import torch
    lens, nq, window, sink, G, H = WAYS[case]
    nq = [m if m else n for m, n in zip(nq, lens)]
    g = gen(300 + case)
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, sum(nq), H * G, d, dtype=dtype).transpose(0, 1)
    k, v = randn(g, H, sum(lens), d, dtype=dtype), randn(g, H, sum(lens), d, dtype=dtype)
    got = binding.sink_attention(q, k, v, window, sink, None, cu_q, cu_k, want_lse=True)
    # some rows of some heads: the first and the last of every sequence, and a spread between
    for s, (m, n) in enumerate(zip(nq, lens)):
        rows = torch.tensor(sorted({0, m - 1, *(int(x) for x in np.linspace(0, m - 1, 23))}), device="cuda")
        seen = ref.seen_by(m, n, window, sink).cuda()[rows]
        a, x = int(cu_q[s]), int(cu_k[s])
        for h in (0, H * G - 1):
            o, e, mass, size = ref.softmax_rows(q[h, a + rows].double(), k[h // G, x:x + n].double(),
                                                v[h // G, x:x + n].double(), seen, d ** -0.5)
            tol, tol_e = ref.attention_bounds(o, e, mass, size, n, d, dtype == "bf16")
            assert bool(((got["out"][h, a + rows].double() - o).abs() <= tol).all()), (s, h)
            assert bool(((got["lse"][h, a + rows].double() - e).abs() <= tol_e).all()), (s, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sink_attention_negative_and_zero_scale(dtype):
    """Any finite scale, on the kernels for few and for many rows."""
    g = gen(41)
    H, G, d, n = 2, 4, 64, 200
    q, k, v = randn(g, H * G, n, d, dtype=dtype), randn(g, H, n, d, dtype=dtype), randn(g, H, n, d, dtype=dtype)
    for m in (2, n):
        for scale in (-0.2, 0.0):
            got = binding.sink_attention(q[:, :m], k, v, 50, 3, scale, [0, m], [0, n], want_lse=True)
            check_attention(got["out"], q[:, :m], k, v, [0, m], [0, n], lambda s, h, i, j: ref.seen_by(i, j, 50, 3), scale,
                            dtype, got["lse"], heads=[0, 7])


def test_sink_attention_split_unseen_values_do_not_matter():
    """As above where a chunk's keys are split over workgroups (bf16, many rows; fp32, few)."""
    import torch
    for dtype, m in (("bf16", 130), ("f32", 3)):
        g = gen(43)
        H, G, d, n, W, sink = 1, 4, 128, 6000, 4000, 4
        q, k, v = randn(g, H * G, m, d, dtype=dtype), randn(g, H, n, d, dtype=dtype), randn(g, H, n, d, dtype=dtype)
        clean = binding.sink_attention(q, k, v, W, sink, None, [0, m], [0, n])["out"]
        seen = ref.seen_by(m, n, W, sink).cuda()
        for j in (2, 900, n - m - W + 1, n - m + 1, n - 1):
            v2 = v.clone()
            v2[:, j, 77] = math.inf
            got = binding.sink_attention(q, k, v2, W, sink, None, [0, m], [0, n])["out"]
            hit = torch.zeros((H * G, m, d), dtype=torch.bool, device="cuda")
            hit[:, seen[:, j], 77] = True
            assert torch.equal(got[~hit], clean[~hit]), (dtype, j)
            assert not bool(torch.isfinite(got[hit]).any()), (dtype, j)


# ---------------------------------------------------------------- together, and far into memory

def test_example_layer():
    """The example's calls in a row: the steps attend over exactly the rows that were kept, then the new ones."""
    import torch
    from paper_2608_27128_amd.examples import serve_layer
    g = gen(47)
    layer = serve_layer.Layer([900, 333], steps=5, n_heads=2, group=4, d=128, window=128)
    T = int(layer.cu[-1])
    q, k, v = serve_layer.projections(T, layer, g)
    got = layer.prompt(q, k, v, torch.rand((2, T), generator=g, device="cuda"))
    assert bool((got["status"] == OK).all()) and layer.length.tolist() == [layer.budget.tolist()] * 2
    want_k = ref.norm_rope(k.transpose(0, 1).double(), layer.k_weight, serve_layer.EPS, layer.rope, layer.positions)
    check_rope(got["keys"], want_k, 128, "bf16")
    qr = binding.qk_norm_rope(q.transpose(0, 1), None, layer.q_weight, None, serve_layer.EPS, layer.rope,
                              layer.positions)["q"]
    check_attention(got["out"].transpose(0, 1), qr, got["keys"], v.transpose(0, 1), layer.cu, layer.cu,
                    lambda s, h, m, n: ref.seen_by(m, n, 128, 4), layer.scale, "bf16", heads=[0, 7])
    for t in range(5):
        q1, k1, v1 = serve_layer.projections(2, layer, g)
        out = layer.step(q1, k1, v1)
        n = layer.length
        assert bool((out["status"] == OK).all()) and n.tolist() == [(layer.budget + t + 1).tolist()] * 2
        kv = binding.cache4_read(layer.cache, n, torch.float32)
        for s in range(2):
            r0 = int(layer.cache.cu_rows[s])
            for h in range(2):
                a = int(layer.cu[s])
                pos = got["s1"][h, a:int(layer.cu[s + 1])].nonzero().squeeze(1)
                kept = ref.quantise(got["keys"][h, a + pos].double())[0]
                assert torch.equal(kv["keys"][h, r0:r0 + len(pos)].double(), kept)
                last = r0 + int(n[h, s]) - 1
                assert torch.equal(kv["values"][h, last].double(), ref.quantise(v1[s, h].double())[0])
        check_attention(out["out"].transpose(0, 1), out["q"], kv["keys"], kv["values"], [0, 1, 2], layer.cache.cu_rows,
                        lambda s, h, m, c: (torch.arange(c)[None, :] < int(n[h // 4, s])).expand(m, c), layer.scale, "bf16")


def test_rows_beyond_32_bits():
    """Byte offsets past 2^32 in keys, values and the 4-bit cache: the last rows of a long buffer."""
    import torch
    g = gen(53)
    H, d, far, n = 2, 128, 9_000_000, 700
    big = torch.empty((H, far + n, d), dtype=torch.bfloat16, device="cuda")   # 2.3 GB a head
    k, v = randn(g, H, n, d), randn(g, H, n, d)
    cu = [0, far, far + n]
    q = randn(g, H * 4, 3, d)
    big[:, far:] = k
    vals = torch.empty_like(big)
    vals[:, far:] = v
    for m in (3, 300):
        q = randn(g, H * 4, m, d)
        got = binding.sink_attention(q, big, vals, 1 << 20, 0, None, [0, 0, m], cu)["out"]
        assert torch.equal(got, binding.sink_attention(q, k, v, 1 << 20, 0, None, [0, m], [0, n])["out"])
    out = binding.qk_norm_rope(None, big[:, far:], None, torch.ones(d, device="cuda"), 1e-6, table(n, d),
                               torch.arange(n, dtype=torch.int32, device="cuda"))["k"]
    check_rope(out, ref.norm_rope(k.double(), torch.ones(d, device="cuda"), 1e-6, table(n, d), torch.arange(n, device="cuda")), d, "bf16")
    ret = torch.zeros((H, far + n), dtype=torch.uint8, device="cuda")
    ret[:, far:] = 1
    rows = 40_000_000                                                        # 2.6 GB of codes a head
    cache = binding.Cache4.empty(H, [rows, n + 1], d)
    kept = binding.cache4_compact(big, vals, ret, cache, cu)
    del big, vals, ret
    assert kept["len"].tolist() == [[0, n]] * H
    small = binding.Cache4.empty(H, [n + 1], d)
    ones = torch.ones((H, n), dtype=torch.uint8, device="cuda")
    near = binding.cache4_compact(k, v, ones, small)
    k1, v1, q1 = randn(g, H, 1, d), randn(g, H, 1, d), randn(g, H * 4, 1, d)
    length = binding.cache4_append(k1, v1, cache, kept["len"], [0, 0, 1])["len"]
    length1 = binding.cache4_append(k1, v1, small, near["len"], [0, 1])["len"]
    a = binding.cache4_attention(q1, cache, length, None, [0, 0, 1])["out"]
    b = binding.cache4_attention(q1, small, length1, None, [0, 1])["out"]
    assert torch.equal(a, b)
    x = binding.cache4_read(cache, length, torch.bfloat16, cu_out=[0, 0, n + 1])
    y = binding.cache4_read(small, length1, torch.bfloat16, cu_out=[0, n + 1])
    for name in ("keys", "values"):
        assert torch.equal(x[name], y[name])


def test_outputs_whose_heads_overlap_are_refused():
    import torch
    g = gen(900)
    H, T, d = 2, 8, 128
    q, k, v = randn(g, H * 2, T, d), randn(g, H, T, d), randn(g, H, T, d)
    one = torch.zeros((1, T, d), dtype=q.dtype, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        binding.qk_norm_rope(q, None, q_out=one.expand(H * 2, T, d))
    with pytest.raises(ValueError, match="overlap"):
        binding.qk_norm_rope(None, k, k_out=one.expand(H, T, d))
    with pytest.raises(ValueError, match="overlap"):
        binding.sink_attention(q, k, v, 4, out=one.expand(H * 2, T, d))
    cache = binding.Cache4.empty(H, [32], d)
    kept = binding.cache4_compact(k, v, torch.ones((H, T), dtype=torch.uint8, device="cuda"), cache)
    with pytest.raises(ValueError, match="overlap"):
        binding.cache4_attention(q, cache, kept["len"], out=one.expand(H * 2, T, d))
    # an input may repeat one head: the same answer as with the copies laid out
    got = binding.sink_attention(q, k[:1].expand(H, T, d), v[:1].expand(H, T, d), 4)["out"]
    want = binding.sink_attention(q, k[:1].repeat(H, 1, 1), v[:1].repeat(H, 1, 1), 4)["out"]
    assert torch.equal(got, want)


# fp32 with rows enough that workgroups of four row tiles go over keys of their own: a ragged batch with sinks that
# end inside a tile, plain causal, rows before the first key, a window of no key but the row's own, many short ones
WIDE = [((400, 1, 0, 37, 350, 600), (400, 1, 0, 37, 100, 600), 90, 33, 3), ((1100,), (1100,), 1 << 40, 0, 4),
        ((300,) * 6, (350,) * 6, 1 << 20, 0, 4), ((900,), (900,), 1, 0, 4), ((70, 65, 64, 63, 1) * 8,) * 2 + (1 << 20, 0, 5),
        ((1200,), (700,), 0, 70, 4)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(WIDE)))
def test_sink_attention_wide_fp32(case, d):
    lens, nq, window, sink, G = WIDE[case]
    g = gen(500 + case)
    H = 8
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, H * G, sum(nq), d, dtype="f32")
    k, v = randn(g, H, sum(lens), d, dtype="f32"), randn(g, H, sum(lens), d, dtype="f32")
    got = binding.sink_attention(q, k, v, window, sink, None, cu_q, cu_k, want_lse=True)
    check_attention(got["out"], q, k, v, cu_q, cu_k, lambda s, h, m, n: ref.seen_by(m, n, window, sink), d ** -0.5,
                    "f32", got["lse"], heads=[0, G, H * G - 1])


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_sink_attention_wide_fp32_unseen_values_do_not_matter(bad):
    import torch
    g = gen(520)
    H, G, d, n, W, sink = 8, 4, 128, 600, 64, 4
    q, k, v = randn(g, H * G, n, d, dtype="f32"), randn(g, H, n, d, dtype="f32"), randn(g, H, n, d, dtype="f32")
    clean = binding.sink_attention(q, k, v, W, sink)["out"]
    seen = ref.seen_by(n, n, W, sink).cuda()
    for j in (2, 17, 300, n - 1):
        v2 = v.clone()
        v2[:, j, 77] = bad
        got = binding.sink_attention(q, k, v2, W, sink)["out"]
        hit = torch.zeros((H * G, n, d), dtype=torch.bool, device="cuda")
        hit[:, seen[:, j], 77] = True
        assert torch.equal(got[~hit], clean[~hit]), j
        assert not bool(torch.isfinite(got[hit]).any()), j


def test_sink_attention_wide_fp32_in_a_graph():
    """Recorded and replayed after other work, on another stream's tensors."""
    import torch
    g = gen(521)
    H, G, d, n = 8, 4, 64, 500
    q, k, v = randn(g, H * G, n, d, dtype="f32"), randn(g, H, n, d, dtype="f32"), randn(g, H, n, d, dtype="f32")
    out = torch.empty_like(q)
    binding.sink_attention(q, k, v, 100, 4, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.sink_attention(q, k, v, 100, 4, out=out)
    for t in range(3):
        q.copy_(randn(g, H * G, n, d, dtype="f32"))
        want = binding.sink_attention(q, k, v, 100, 4)["out"]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), t
