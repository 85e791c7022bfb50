"""Accumulated attention weights, the 8-bit cache, attention over it and eviction from it on the GPU, against plain
64-bit forms (cache8_ref.py, cache_ops_ref.py).  Tolerances are those that the number formats give; the 8-bit values
and the kept rows are exact."""
import math

import numpy as np
import pytest

import cache8_ref as ref8
import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache_ops import ATTN, check_attention, cum, gen, randn

pytestmark = pytest.mark.gpu
OK, MISMATCH, NONFINITE = 0, 1, 2


# ---------------------------------------------------------------- accumulated weights

def lse_of(q, k, cu_q, cu_k, window, sink, scale):
    """The queries' log-sum-exp in 64 bits, rounded once."""
    import torch
    Hq, Tq, _ = q.shape
    G = Hq // k.shape[0]
    lse = torch.full((Hq, Tq), -math.inf, dtype=torch.float64, device=q.device)
    for s in range(len(cu_q) - 1):
        a, b, x, y = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        if a == b or x == y:
            continue
        seen = ref.seen_by(b - a, y - x, window, sink).to(q.device)
        for h in range(Hq):
            z = (q[h, a:b].double() @ k[h // G, x:y].double().T) * scale
            lse[h, a:b] = torch.logsumexp(z.masked_fill(~seen, -math.inf), 1)
    return lse.float()


def check_mass(got, q, k, lse, cu_q, cu_k, seen_of, scale, before=None):
    Hq, _, d = q.shape
    H = k.shape[0]
    G = Hq // H
    for s in range(len(cu_q) - 1):
        a, b, x, y = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        for h in range(H):
            seen = seen_of(s, h, b - a, y - x).to(q.device)
            hs = slice(h * G, h * G + G)
            want, tol = ref8.mass_of(q[hs, a:b].double(), k[h, x:y].double(), lse[hs, a:b].double(), seen, scale,
                                     None if before is None else before[h, x:y].double())
            err = (got[h, x:y].double() - want).abs()
            assert bool((err <= tol).all()), (s, h, float((err - tol).max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention_mass(case, dtype, d):
    lens, nq, window, sink, G = ATTN[case]
    nq = [m if m else (n if len(lens) == 1 else 0) for m, n in zip(nq, lens)]
    g = gen(300 + case)
    H = 2
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, H * G, sum(nq), d, dtype=dtype)
    k = randn(g, H, sum(lens), d, dtype=dtype) + 2 * randn(g, H, 1, d, dtype=dtype)
    lse = lse_of(q, k, cu_q, cu_k, window, sink, d ** -0.5)
    got = binding.attention_mass(q, k, lse, window, sink, None, cu_q, cu_k)["mass"]
    check_mass(got, q, k, lse, cu_q, cu_k, lambda s, h, m, n: ref.seen_by(m, n, window, sink), d ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk,G", [(3000, 300, 8), (3000, 900, 1), (700, 129, 20), (5000, 5000, 1)])
def test_attention_mass_split_rows(nq, nk, G, dtype):
    """Few keys and many rows, some of them before the first key: the rows are split over workgroups and joined."""
    import torch
    g = gen(nq + nk + G)
    q, k = randn(g, G, nq, 64, dtype=dtype), randn(g, 1, nk, 64, dtype=dtype)
    lse = lse_of(q, k, [0, nq], [0, nk], nk, 0, 0.125)
    assert binding.lib().twinkv_mass_workspace_bytes(0 if dtype == "bf16" else 1, 64, 1, G, 1, binding._i64_array([0, nq]),
                                                     binding._i64_array([0, nk]), nk, 0) > 0
    got = binding.attention_mass(q, k, lse, nk, 0, 0.125)["mass"]
    check_mass(got, q, k, lse, [0, nq], [0, nk], lambda s, h, m, n: ref.seen_by(m, n, nk, 0), 0.125)
    again = binding.attention_mass(q, k, lse, nk, 0, 0.125)["mass"]
    assert torch.equal(got, again)


def test_attention_mass_adds_up_over_chunks():
    """A prompt's chunks, each added to what the earlier ones gave, in place; and the whole prompt at once."""
    import torch
    g = gen(21)
    T, H, G, d, cut = 700, 2, 4, 128, 333
    qkv = randn(g, T, H * G + H, d)                       # token major, as a projection leaves it
    q, k = (x.transpose(0, 1) for x in qkv.split([H * G, H], 1))
    full = binding.sink_attention(q, k, k, T, 0, want_lse=True)["lse"]
    whole = binding.attention_mass(q, k, full, T, 0)["mass"]
    check_mass(whole, q, k, full, [0, T], [0, T], lambda s, h, m, n: ref.seen_by(m, n, T, 0), d ** -0.5)
    acc = torch.zeros((H, T), device="cuda")
    first = binding.attention_mass(q[:, :cut], k[:, :cut], full[:, :cut].contiguous(), T, 0)["mass"]
    acc[:, :cut] = first
    before = acc.clone()
    got = binding.attention_mass(q[:, cut:], k, full[:, cut:].contiguous(), T, 0, mass=acc, out=acc)["mass"]
    assert got.data_ptr() == acc.data_ptr()
    check_mass(acc, q[:, cut:], k, full[:, cut:], [0, T - cut], [0, T], lambda s, h, m, n: ref.seen_by(m, n, T, 0),
               d ** -0.5, before)
    # every query's weights sum to 1: G T in all
    assert abs(float(whole.double().sum()) / (H * G * T) - 1) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_mass_unseen_keys_do_not_matter(dtype):
    """A NaN key spoils its own sum alone, rows whose log-sum-exp is -inf weigh nothing, and a NaN query reaches the
    keys that it sees."""
    import torch
    g = gen(31)
    n, H, G, d, W, sink = 500, 2, 3, 128, 40, 3
    q, k = randn(g, H * G, n, d, dtype=dtype), randn(g, H, n, d, dtype=dtype)
    lse = lse_of(q, k, [0, n], [0, n], W, sink, 0.1)
    clean = binding.attention_mass(q, k, lse, W, sink, 0.1)["mass"]
    k2 = k.clone()
    k2[0, 77] = math.nan
    k2[1, 2, 5] = math.inf
    got = binding.attention_mass(q, k2, lse, W, sink, 0.1)["mass"]
    rest = torch.ones_like(clean, dtype=torch.bool)
    rest[0, 77] = rest[1, 2] = False
    assert torch.equal(got[rest], clean[rest]) and math.isnan(float(got[0, 77]))
    q2 = q.clone()
    q2[1, 300] = math.nan
    got = binding.attention_mass(q2, k, lse, W, sink, 0.1)["mass"]
    seen = ref.seen_by(n, n, W, sink)[300].cuda()
    assert bool(torch.isnan(got[0][seen]).all()) and torch.equal(got[0][~seen], clean[0][~seen])
    assert torch.equal(got[1], clean[1])
    none = lse.clone()
    none[2, 100:140] = -math.inf
    got = binding.attention_mass(q, k, none, W, sink, 0.1)["mass"]
    check_mass(got, q, k, none, [0, n], [0, n], lambda s, h, m, nk: ref.seen_by(m, nk, W, sink), 0.1)


def test_attention_mass_long_sums():
    """200000 rows on 40 keys: the sums keep their digits."""
    g = gen(33)
    G, m, d = 8, 25000, 64
    q, k = randn(g, G, m, d), randn(g, 1, 40, d)
    lse = lse_of(q, k, [0, m], [0, 40], 1 << 40, 0, 0.125)
    got = binding.attention_mass(q, k, lse, 1 << 40, 0, 0.125)["mass"]
    want, _ = ref8.mass_of(q.double(), k[0].double(), lse.double(), ref.seen_by(m, 40, 1 << 40, 0).cuda(), 0.125)
    assert float(((got[0].double() - want).abs() / want).max()) < 1e-6


def test_attention_mass_no_queries_and_no_keys():
    import torch
    k = torch.zeros((2, 5, 64), device="cuda")
    q = torch.zeros((4, 0, 64), device="cuda")
    lse = torch.zeros((4, 0), device="cuda")
    old = torch.arange(10.0, device="cuda").reshape(2, 5)
    assert torch.equal(binding.attention_mass(q, k, lse, 5, 0, mass=old)["mass"], old)
    assert not bool(binding.attention_mass(q, k, lse, 5, 0)["mass"].any())
    q1, lse1 = torch.ones((4, 3, 64), device="cuda"), torch.full((4, 3), -math.inf, device="cuda")
    assert binding.attention_mass(q1, k[:, :0], lse1, 5, 0)["mass"].shape == (2, 0)
    assert not bool(binding.attention_mass(q1, k, lse1, 0, 0)["mass"].any())


def test_attention_mass_many_sequences():
    """More sequences than the kernel arguments hold: the words go through the workspace."""
    g = gen(17)
    S, H, G, d = 400, 1, 2, 64
    lens = [(i * 37) % 50 for i in range(S)]
    nq = [min(n, 1 + i % 3) for i, n in enumerate(lens)]
    cu_q, cu_k = cum(nq), cum(lens)
    q, k = randn(g, H * G, int(cu_q[-1]), d), randn(g, H, int(cu_k[-1]), d)
    lse = lse_of(q, k, cu_q, cu_k, 20, 2, d ** -0.5)
    got = binding.attention_mass(q, k, lse, 20, 2, None, cu_q, cu_k)["mass"]
    check_mass(got, q, k, lse, cu_q, cu_k, lambda s, h, m, n: ref.seen_by(m, n, 20, 2), d ** -0.5)


# ---------------------------------------------------------------- writing and reading the cache

def poison(cache):
    """Rows not in use may hold anything."""
    cache.k_codes.fill_(-128)
    cache.v_codes.fill_(-128)
    cache.k_scales.fill_(255)
    cache.v_scales.fill_(255)
    return cache


def check_rows(cache, length, want, dtype):
    """want[h][s] = (keys, values) float64 of the rows in use."""
    import torch
    kv = binding.cache8_read(cache, length, dtype)
    for h in range(cache.n_heads):
        for s in range(cache.n_seqs):
            r0, r1 = int(cache.cu_rows[s]), int(cache.cu_rows[s + 1])
            n = int(length[h, s])
            for name, x in zip(("keys", "values"), want[h][s]):
                assert len(x) == n, (h, s, name)
                assert torch.equal(kv[name][h, r0:r0 + n].double(), x), (h, s, name)
                assert not bool(kv[name][h, r0 + n:r1].any()), (h, s, name)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,spare", [((100,), 0), ((1, 0, 33, 515), 40), ((6011,), 7)])
def test_cache8_compact(lens, spare, dtype, d):
    import torch
    g = gen(sum(lens) + d)
    H, T, cu = 3, sum(lens), cum(lens)
    keys = randn(g, T, H, d, dtype=dtype).transpose(0, 1) * 3
    values = randn(g, H, T, d, dtype=dtype)
    keys[0, :, :8] *= 1e-3
    values[1, ::3] *= 1e4
    values[2, ::5] = 0
    ret = (torch.rand((H, T), generator=g, device="cuda") < 0.4).to(torch.uint8) * 7  # any nonzero byte keeps
    mass = torch.rand((H, T), generator=g, device="cuda")
    caps = [int(ret[:, a:b].ne(0).sum(1).max()) + spare if b > a else 0 for a, b in zip(cu[:-1], cu[1:])]
    cache = poison(binding.Cache8.empty(H, caps, d))
    got = binding.cache8_compact(keys, values, ret, cache, cu, token_mass=mass)
    assert bool((got["status"] == OK).all())
    want = []
    for h in range(H):
        want.append([])
        for s in range(len(lens)):
            a, b, r0, r1 = int(cu[s]), int(cu[s + 1]), int(cache.cu_rows[s]), int(cache.cu_rows[s + 1])
            pos = ret[h, a:b].nonzero().squeeze(1)
            n = len(pos)
            assert int(got["len"][h, s]) == n
            assert torch.equal(got["pos"][h, r0:r0 + n].long(), pos)
            assert bool((got["pos"][h, r0 + n:r1] == -1).all())
            assert torch.equal(got["mass"][h, r0:r0 + n], mass[h, a + pos])
            assert not bool(got["mass"][h, r0 + n:r1].any())
            want[h].append([ref8.stored(x[h, a + pos].double())[0] for x in (keys, values)])
    check_rows(cache, got["len"], want, keys.dtype)


def test_cache8_every_bf16():
    """Every bf16 number, in a block of its own (largest and alone), and beside one half as large as the largest."""
    import torch
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16)
    rows = torch.zeros((1, 65536 * 32, 64), dtype=torch.bfloat16, device="cuda")
    rows[0, ::32, 0] = x
    rows[0, 1::32, 7] = 0.5 * x
    rows[0, 2::32, 9] = 0.01 * x
    cache = binding.Cache8.empty(1, 65536 * 32, 64)
    ones = torch.ones((1, 65536 * 32), dtype=torch.uint8, device="cuda")
    got = binding.cache8_compact(rows, rows, ones, cache)
    assert int(got["status"]) == NONFINITE
    kv = binding.cache8_read(cache, got["len"], torch.float32)
    v = rows[0].reshape(65536, 32 * 64).double()
    v = torch.where(torch.isfinite(rows[0].double()).all(-1).reshape(65536, 32).repeat_interleave(64, 1), v, 0.0)
    top = v.abs().amax(1, keepdim=True)
    byte = torch.full_like(top, 248.0)
    for b in range(248, 0, -1):
        byte = torch.where(top < 127.5 * 2.0 ** (b - 127), torch.full_like(byte, float(b)), byte)
    grid = ((byte.long() + 896) << 52).view(torch.float64)   # 2^(byte - 127), exactly
    want = (torch.round(v / grid).clamp(-127, 127) * grid).reshape(-1, 64)
    assert torch.equal(kv["keys"][0].double(), want)
    assert torch.equal(kv["values"][0].double(), want)


def test_cache8_states():
    """A problem that keeps more than its rows stores nothing; a row that is not finite is zeros and reported, and the
    rows beside it are as without it."""
    import torch
    g = gen(5)
    H, d, lens = 2, 128, (100, 60)
    cu, T = cum(lens), 160
    keys, values = randn(g, H, T, d), randn(g, H, T, d)
    ret = torch.ones((H, T), dtype=torch.uint8, device="cuda")
    ret[0, 40:100] = 0
    keys[0, 120, 70] = math.inf
    values[0, 121, 3] = math.nan
    cache = poison(binding.Cache8.empty(H, [64, 64], d))
    got = binding.cache8_compact(keys, values, ret, cache, cu)
    assert got["len"].tolist() == [[40, 60], [0, 60]]
    assert got["status"].tolist() == [[OK, NONFINITE], [MISMATCH, OK]]
    assert bool((got["pos"][1, :64] == -1).all())
    empty = torch.zeros((0, d), dtype=torch.float64, device="cuda")
    want = [[[empty, empty] if (h, s) == (1, 0) else
             [ref8.stored(x[h, int(cu[s]):int(cu[s]) + int(got["len"][h, s])].double())[0] for x in (keys, values)]
             for s in range(2)] for h in range(H)]
    check_rows(cache, got["len"], want, torch.bfloat16)
    assert not bool(want[0][1][0][20].any()) and bool(want[0][1][1][20].any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache8_append(dtype, d):
    """Rows one by one, a few, a block's worth, and more than one wave writes; with growing and falling magnitudes, so
    that blocks are rounded again; lengths that differ from head to head; in place."""
    import torch
    g = gen(41)
    H, S = 3, 2
    cache = poison(binding.Cache8.empty(H, [640, 320], d))
    length = torch.zeros((H, S), dtype=torch.int32, device="cuda")
    want = [[[ref8.Rows8(d, "cuda"), ref8.Rows8(d, "cuda")] for _ in range(S)] for _ in range(H)]
    # (so that heads differ) head 0 begins with rows of its own
    mags = [1.0, 0.3, 5.0, 2.0, 100.0, 1e-4, 7e3, 1.0]
    counts = [(1, 0), (1, 1), (1, 2), (3, 1), (30, 5), (1, 31), (40, 32), (64, 0), (129, 1), (200, 140), (0, 0), (1, 1)]
    for i, new in enumerate(counts):
        cu = cum(new)
        T = int(cu[-1])
        k, v = (randn(g, T, H, d, dtype=dtype).transpose(0, 1) * mags[(i + x) % len(mags)] for x in (0, 3))
        if i == 4:
            k[1, 2] = math.nan
        got = binding.cache8_append(k, v, cache, length, cu, len_out=length)
        assert got["len"].data_ptr() == length.data_ptr()
        for h in range(H):
            for s in range(S):
                a, b = int(cu[s]), int(cu[s + 1])
                bad = [w.append(x[h, a:b].double()) for w, x in zip(want[h][s], (k, v))]
                assert int(got["status"][h, s]) == (NONFINITE if any(bad) else OK), (i, h, s)
        assert length.tolist() == [[sum(c[s] for c in counts[:i + 1]) for s in range(S)]] * H
        check_rows(cache, length, [[[w.x for w in want[h][s]] for s in range(S)] for h in range(H)], k.dtype)


@pytest.mark.parametrize("many", [False, True])
def test_cache8_append_does_not_fit(many):
    """A problem whose new tokens do not fit, or whose length is negative, stays as it is; the others grow."""
    import torch
    g = gen(43)
    H, d, n = 4, 64, 200 if many else 3
    cache = poison(binding.Cache8.empty(H, [224], d))
    k, v = randn(g, H, n, d), randn(g, H, n, d)
    length = torch.tensor([[224 - n], [224 - n + 1], [-1], [0]], dtype=torch.int32, device="cuda")
    before = [x.clone() for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    got = binding.cache8_append(k, v, cache, length)
    assert got["len"].tolist() == [[224], [224 - n + 1], [-1], [n]]
    assert got["status"].tolist() == [[OK], [MISMATCH], [MISMATCH], [OK]]
    for x, y in zip(before, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)):
        assert torch.equal(x[1:3], y[1:3])
    kv = binding.cache8_read(cache, got["len"], torch.float32, want_values=False)
    assert sorted(kv) == ["keys"]
    assert torch.equal(kv["keys"][3, :n].double(), ref8.stored(k[3].double())[0])


def filled(g, H, rows, d, dtype="bf16", lens=None):
    """A cache of random rows, some of them larger, its lengths (a few less in each head), and its values in fp32."""
    import torch
    cache = poison(binding.Cache8.empty(H, rows, d))
    C, cu = int(cache.cu_rows[-1]), cache.cu_rows
    k, v = randn(g, H, C, d, dtype=dtype) + 2 * randn(g, H, 1, d, dtype=dtype), randn(g, H, C, d, dtype=dtype)
    v[:, ::37] *= 30
    if lens is None:
        lens = [[max(0, int(n) - 3 * h) for n in rows] for h in range(H)]
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    use = torch.zeros((H, C), dtype=torch.uint8, device="cuda")
    for h in range(H):
        for s in range(len(rows)):
            use[h, int(cu[s]):int(cu[s]) + lens[h][s]] = 1
    got = binding.cache8_compact(k, v, use, cache, cu)
    assert torch.equal(got["len"], length)
    kv = binding.cache8_read(cache, length, torch.float32)
    return cache, length, kv["keys"], kv["values"]


def test_cache8_read_parts():
    """Any first row and count; rows outside those in use are zeros."""
    import torch
    g = gen(47)
    H, d = 2, 64
    cache, length, keys, _ = filled(g, H, [100, 70], d)
    first = torch.tensor([[0, -5], [33, 64]], dtype=torch.int32, device="cuda")
    cu_out = [0, 110, 150]
    got = binding.cache8_read(cache, length, torch.bfloat16, first, cu_out)
    for h in range(H):
        for s in range(2):
            for r in range(cu_out[s + 1] - cu_out[s]):
                x = int(first[h, s]) + r
                want = keys[h, int(cache.cu_rows[s]) + x] if 0 <= x < int(length[h, s]) else torch.zeros(d, device="cuda")
                assert torch.equal(got["keys"][h, cu_out[s] + r].float(), want), (h, s, r)


# ---------------------------------------------------------------- attention over the cache

ATTN8 = [  # rows, queries, group
    ((1,), (1,), 1), ((5,), (1,), 4), ((31,), (3,), 4), ((64,), (64,), 1), ((100,), (7,), 5), ((513,), (1,), 4),
    ((700,), (2,), 16), ((40, 0, 1, 333, 64), (1, 1, 2, 0, 5), 3), ((2000,), (9,), 8), ((3, 5000), (1, 1), 4),
    ((1100,), (70,), 4), ((9000,), (1,), 2)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(ATTN8)))
def test_cache8_attention(case, dtype, d):
    """out, lse and the rows' weights; queries that see nothing; lengths that differ from head to head."""
    import torch
    rows, nq, G = ATTN8[case]
    g = gen(500 + case)
    H = 2
    cache, length, keys, values = filled(g, H, rows, d, dtype)
    cu_q, cu = cum(nq), cache.cu_rows
    q = randn(g, int(cu_q[-1]), H * G, d, dtype=dtype).transpose(0, 1)
    old = torch.rand(keys.shape[:2], generator=g, device="cuda")
    got = binding.cache8_attention(q, cache, length, None, cu_q, want_lse=True, mass=old)
    alone = binding.cache8_attention(q, cache, length, None, cu_q)
    assert sorted(alone) == ["out"] and torch.equal(alone["out"], got["out"])
    for s in range(len(rows)):
        a, b = int(cu_q[s]), int(cu_q[s + 1])
        for h in range(H):
            n, r0, r1 = int(length[h, s]), int(cu[s]), int(cu[s + 1])
            k, v = keys[h, r0:r0 + n], values[h, r0:r0 + n]
            seen = ref.seen_by(b - a, n, 1 << 40, 0)
            for x in sorted({0, G - 1}):
                check_attention(got["out"][h * G + x:h * G + x + 1, a:b], q[h * G + x:h * G + x + 1, a:b], k[None], v[None],
                                [0, b - a], [0, n], lambda *_: seen, d ** -0.5, dtype,
                                got["lse"][h * G + x:h * G + x + 1, a:b])
            hs = slice(h * G, h * G + G)
            check_mass(got["mass"][None, h, r0:r0 + n], q[hs, a:b], k[None], got["lse"][hs, a:b], [0, b - a], [0, n],
                       lambda *_: seen, d ** -0.5, old[None, h, r0:r0 + n])
            assert not bool(got["mass"][h, r0 + n:r1].any())


def test_cache8_attention_mass_in_place_and_from_nothing():
    import torch
    g = gen(61)
    H, G, d = 2, 4, 128
    cache, length, _, _ = filled(g, H, [300, 90], d)
    q = randn(g, H * G, 2, d)
    cu_q = [0, 1, 2]
    first = binding.cache8_attention(q, cache, length, None, cu_q, want_mass=True)
    zero = binding.cache8_attention(q, cache, length, None, cu_q, mass=torch.zeros_like(first["mass"]))
    assert torch.equal(first["mass"], zero["mass"])
    acc = first["mass"].clone()
    want = binding.cache8_attention(q, cache, length, None, cu_q, mass=first["mass"])["mass"]
    got = binding.cache8_attention(q, cache, length, None, cu_q, mass=acc, mass_out=acc)["mass"]
    assert got.data_ptr() == acc.data_ptr() and torch.equal(acc, want)
    # a query's weights over its rows sum to 1
    assert abs(float(first["mass"][:, :320].double().sum()) / (H * G) - 1) < 1e-5
    # no queries: what was there, on the rows in use
    none = binding.cache8_attention(q[:, :0], cache, length, None, [0, 0, 0], mass=acc)["mass"]
    assert torch.equal(none, acc)


def test_cache8_attention_many_sequences_and_long_rows():
    """More sequences than the kernel arguments hold; one long cache among short ones."""
    g = gen(67)
    S, H, G, d = 300, 1, 2, 64
    rows = [(i * 37) % 90 for i in range(S)]
    rows[150] = 20000
    cache, length, keys, values = filled(g, H, rows, d)
    cu_q = cum([1] * S)
    q = randn(g, H * G, S, d)
    got = binding.cache8_attention(q, cache, length, None, cu_q, want_lse=True, want_mass=True)
    for s in [0, 1, 2, 3, 77, 149, 150, 151, 299]:
        n, r0 = int(length[0, s]), int(cache.cu_rows[s])
        k, v = keys[:, r0:r0 + n], values[:, r0:r0 + n]
        seen = ref.seen_by(1, n, 1 << 40, 0)
        check_attention(got["out"][:, s:s + 1], q[:, s:s + 1], k, v, [0, 1], [0, n], lambda *_: seen, d ** -0.5, "bf16",
                        got["lse"][:, s:s + 1])
        check_mass(got["mass"][:, r0:r0 + n], q[:, s:s + 1], k, got["lse"][:, s:s + 1], [0, 1], [0, n], lambda *_: seen,
                   d ** -0.5)


# ---------------------------------------------------------------- eviction

EVICT = [  # rows, budgets, sinks, recent
    ((100,), (60,), 4, 16), ((100,), (100,), 4, 16), ((64,), (0,), 0, 0), ((1,), (1,), 4, 64), ((300, 0, 33, 40), (100, 0, 33, 7), 4, 16),
    ((5000,), (4900,), 4, 64), ((5000,), (321,), 0, 0), ((17000,), (9000,), 4, 64), ((900,), (20,), 30, 30)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_cache8_evict(case, d):
    """The kept rows, their order, positions and weights exactly, and their values in the new blocks."""
    import torch
    rows, budget, sink, recent = EVICT[case]
    g = gen(700 + case)
    H = 2
    cache, length, keys, values = filled(g, H, rows, d)
    C = keys.shape[1]
    mass = (torch.rand((H, C), generator=g, device="cuda") * 50).floor() / 8          # many ties
    mass[0, ::11] = math.nan
    mass[0, 5::97] = math.inf
    mass[1, 3::29] = -0.0
    mass[1, 4::29] = 0.0
    mass[1, 7::31] = -1.5
    pos = torch.randint(-5, 1 << 30, (H, C), generator=g, device="cuda", dtype=torch.int32)
    to = poison(binding.Cache8.empty(H, [b + 20 for b in budget], d))
    for p in (pos, None):
        got = binding.cache8_evict(cache, length, mass, budget, to, sink, recent, pos=p)
        want = []
        for h in range(H):
            want.append([])
            for s in range(len(rows)):
                n, r0, t0, t1 = int(length[h, s]), int(cache.cu_rows[s]), int(to.cu_rows[s]), int(to.cu_rows[s + 1])
                kept = torch.tensor(ref8.kept_rows(mass[h, r0:r0 + n].tolist(), n, budget[s], sink, recent),
                                    dtype=torch.int64, device="cuda")
                m = len(kept)
                assert int(got["len"][h, s]) == m
                assert torch.equal(got["pos"][h, t0:t0 + m], kept.int() if p is None else p[h, r0 + kept])
                assert bool((got["pos"][h, t0 + m:t1] == -1).all())
                assert torch.equal(got["mass"][h, t0:t0 + m].view(torch.int32), mass[h, r0 + kept].view(torch.int32))
                assert not bool(got["mass"][h, t0 + m:t1].any())
                want[h].append([ref8.stored(x[h, r0 + kept].double())[0] for x in (keys, values)])
        check_rows(to, got["len"], want, torch.float32)


def test_cache8_evict_is_the_policy_selection():
    """Where all heads have one length, the kept rows are those of select_topk."""
    import torch
    g = gen(71)
    H, d, n = 3, 64, 1000
    cache, length, _, _ = filled(g, H, [n], d, lens=[[n]] * H)
    mass = torch.rand((H, int(cache.cu_rows[-1])), generator=g, device="cuda")
    kept = binding.select_topk(mass[:, :n].contiguous(), 600, n_sink=4, n_recent=64)["retained"]
    to = binding.Cache8.empty(H, 600, d)
    got = binding.cache8_evict(cache, length, mass, 600, to, 4, 64)
    for h in range(H):
        assert torch.equal(got["pos"][h, :600].long(), kept[h].nonzero().squeeze(1))


def test_cache8_evict_clamps_lengths():
    """A length outside its problem's rows is taken as 0 or all of them."""
    import torch
    g = gen(73)
    cache, length, _, _ = filled(g, 2, [96], 64, lens=[[96], [96]])
    bad = torch.tensor([[-7], [1 << 30]], dtype=torch.int32, device="cuda")
    to = poison(binding.Cache8.empty(2, 96, 64))
    got = binding.cache8_evict(cache, bad, torch.ones((2, 96), device="cuda"), 90, to, 0, 0, len_out=bad)
    assert got["len"].tolist() == [[0], [90]] and bool((got["pos"][0] == -1).all())
    assert got["pos"][1].tolist() == list(range(90)) + [-1] * 6
