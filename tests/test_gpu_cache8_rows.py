"""Attention over the 8-bit cache in batches whose plan takes two row tiles a wave, or would if the queries of
sequences without rows decided it (tests/host/cache8_plans_test.cpp holds the plans of these batches to that)."""
import math

import pytest

import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache8 import check_mass, filled
from test_gpu_cache_ops import check_attention, cum, gen, randn

pytestmark = pytest.mark.gpu


def check_problem(got, q, cache, length, keys, values, h, s, cu_q, G, old):
    """One problem's outputs (of its first and last query head), log-sum-exps and weights."""
    a, b, r0, r1 = int(cu_q[s]), int(cu_q[s + 1]), int(cache.cu_rows[s]), int(cache.cu_rows[s + 1])
    n, d = int(length[h, s]), cache.d
    k, v = keys[h, r0:r0 + n], values[h, r0:r0 + n]
    seen = ref.seen_by(b - a, n, 1 << 40, 0)
    for x in sorted({0, G - 1}):
        one = slice(h * G + x, h * G + x + 1)
        check_attention(got["out"][one, a:b], q[one, a:b], k[None], v[None], [0, b - a], [0, n], lambda *_: seen,
                        d ** -0.5, "bf16", got["lse"][one, a:b])
    hs = slice(h * G, h * G + G)
    check_mass(got["mass"][None, h, r0:r0 + n], q[hs, a:b], k[None], got["lse"][hs, a:b], [0, b - a], [0, n],
               lambda *_: seen, d ** -0.5, old[None, h, r0:r0 + n])
    assert not bool(got["mass"][h, r0 + n:r1].any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G,rows,nq", [(16, 8, [131072, 0], [1, 40]), (8, 4, [4096] * 64 + [0], [1] * 64 + [300]),
                                         (8, 8, [4096] * 64 + [0], [1] * 64 + [512])])
def test_weights_beside_queries_without_rows(H, G, rows, nq, d):
    """Few rows a problem, in one split and in many, beside a sequence of many queries and no cached row, which gets
    zeros."""
    import torch
    g = gen(len(rows) + G + d)
    cache, length, keys, values = filled(g, H, rows, d)
    cu_q = cum(nq)
    q = randn(g, H * G, int(cu_q[-1]), d)
    old = torch.rand(keys.shape[:2], generator=g, device="cuda")
    new = torch.full_like(old, math.nan)
    got = binding.cache8_attention(q, cache, length, None, cu_q, want_lse=True, mass=old, mass_out=new)
    for h, s in [(0, 0), (H - 1, 0), (1, len(rows) - 2), (H // 2, (len(rows) - 1) // 2)]:
        check_problem(got, q, cache, length, keys, values, h, s, cu_q, G, old)
    assert bool(torch.isfinite(got["mass"]).all())
    last = int(cu_q[-2])
    assert not bool(got["out"][:, last:].any()) and bool((got["lse"][:, last:] == -math.inf).all())


@pytest.mark.parametrize("d", [64, 128])
def test_two_row_tiles_over_a_long_cache(d):
    """28 rows a problem, the second tile of 12, keys in many splits."""
    import torch
    g = gen(d)
    H, G, nq, rows = 8, 4, 7, 131072
    cache, length, keys, values = filled(g, H, [rows], d, lens=[[rows - 1000 * h - h] for h in range(H)])
    q = randn(g, H * G, nq, d)
    old = torch.rand(keys.shape[:2], generator=g, device="cuda")
    got = binding.cache8_attention(q, cache, length, None, [0, nq], want_lse=True, mass=old)
    alone = binding.cache8_attention(q, cache, length, None, [0, nq], want_lse=True)
    assert torch.equal(alone["out"], got["out"]) and torch.equal(alone["lse"], got["lse"])
    for h in (0, 5, H - 1):
        check_problem(got, q, cache, length, keys, values, h, 0, [0, nq], G, old)


@pytest.mark.parametrize("d", [64, 128])
def test_two_row_tiles_of_many_sequences(d):
    """17 to 40 rows a problem, so that the last tile has 1 to 16; lengths of all kinds, fewer than queries and none
    among them, that differ from head to head; one problem of 32 cached rows."""
    import torch
    g = gen(100 + d)
    H, G, S = 4, 1, 64
    nq, rows = [17 + s % 24 for s in range(S)], [32 if s == 5 else 4096 for s in range(S)]
    lens = [[min(rows[s], [(997 * s + 131 * h) % 4097, 4096, 0, 20, 1][s % 5 if s % 3 else 0]) for s in range(S)]
            for h in range(H)]
    cache, length, keys, values = filled(g, H, rows, d, lens=lens)
    cu_q = cum(nq)
    q = randn(g, H * G, int(cu_q[-1]), d)
    old = torch.rand(keys.shape[:2], generator=g, device="cuda")
    got = binding.cache8_attention(q, cache, length, None, cu_q, want_lse=True, mass=old)
    for s in range(S):
        check_problem(got, q, cache, length, keys, values, s % H, s, cu_q, G, old)
    assert bool(torch.isfinite(got["out"].float()).all()) and bool(torch.isfinite(got["mass"]).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("rows,nq,G", [(300, 3, 4), (9000, 5, 3), (300, 9, 4), (9000, 8, 3)])
def test_weights_of_a_nan_query_reach_the_keys_that_it_sees(rows, nq, G, dtype, d):
    """And no key behind it: with scores kept in one split and in many, and with weights computed afresh."""
    import torch
    g = gen(rows + nq)
    H = 2
    cache, length, _, _ = filled(g, H, [rows], d, dtype)
    q = randn(g, H * G, nq, d, dtype=dtype)
    clean = binding.cache8_attention(q, cache, length, None, [0, nq], want_lse=True, want_mass=True)
    q[1, 0] = math.nan
    q[G, nq - 2, d - 1] = math.nan
    got = binding.cache8_attention(q, cache, length, None, [0, nq], want_lse=True, want_mass=True)
    for h, first in ((0, 0), (1, nq - 2)):
        seen = int(length[h, 0]) - (nq - 1 - first)  # keys that the query sees
        assert bool(torch.isnan(got["mass"][h, :seen]).all())
        assert torch.equal(got["mass"][h, seen:], clean["mass"][h, seen:]) and bool(clean["mass"][h, seen] > 0)


@pytest.mark.parametrize("nq", [1, 9])
def test_outputs_in_the_queries_place(nq):
    """Refused where weights are wanted, which come from the queries after the output is written (36 rows a problem);
    without weights a tile of rows reads its queries before it writes."""
    import torch
    g = gen(nq)
    cache, length, _, _ = filled(g, 2, [3000], 128)
    q = randn(g, 8, nq, 128)
    want = binding.cache8_attention(q, cache, length, None, [0, nq])["out"].clone()
    old = torch.zeros((2, int(cache.cu_rows[-1])), device="cuda")
    for kw in (dict(want_mass=True), dict(mass=old), dict(mass_out=old)):
        same = q.clone()
        with pytest.raises(ValueError, match="may not be q"):
            binding.cache8_attention(same, cache, length, None, [0, nq], out=same, **kw)
        assert torch.equal(same, q)
    assert torch.equal(binding.cache8_attention(same, cache, length, None, [0, nq], out=same)["out"], want)
