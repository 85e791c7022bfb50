"""Edges of the operators around the cache on the GPU, against plain 64-bit forms (cache_ops_ref.py)."""
import math

import numpy as np
import pytest

import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache_ops import check_rope, cum, fill_cache, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_table_without_rows(dtype):
    """Every position lies outside a table of no rows: NaN, not the rows as they are."""
    import torch
    g = gen(1000)
    d, T = 64, 9
    q, k = randn(g, 4, T, d, dtype=dtype), randn(g, 2, T, d, dtype=dtype)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rope = torch.zeros((0, d), device="cuda")
    for w in (None, torch.ones(d, device="cuda")):
        got = binding.qk_norm_rope(q, k, w, w, 1e-6, rope, pos)
        for name in ("q", "k"):
            assert bool(torch.isnan(got[name]).all()), name
    empty = torch.zeros((2, 0, d), device="cuda")
    assert binding.qk_norm_rope(empty, None, rope=rope, positions=pos[:0])["q"].shape == (2, 0, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_rotation_a_channel_is_its_own(dtype, d):
    """No table: what one channel holds, infinities and NaN included, does not reach the channel it would turn
    with, and without a weight either the rows come back bit for bit."""
    import torch
    g = gen(1001)
    T, c = 37, 5
    q, k = randn(g, 5, T, d, dtype=dtype), randn(g, 2, T, d, dtype=dtype)
    for j, what in enumerate((math.inf, -math.inf, math.nan, -0.0)):
        q[:, j, c], k[:, j, c + d // 2] = what, what
    got = binding.qk_norm_rope(q, k)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for name, x in (("q", q), ("k", k)):
        nan = torch.isnan(x)
        assert torch.equal(torch.isnan(got[name]), nan), name
        assert torch.equal(got[name].view(bits)[~nan], x.view(bits)[~nan]), name
    # with a norm an infinity's own row has a mean of infinity: itself NaN, the other channels zeros
    w = torch.ones(d, device="cuda")
    got = binding.qk_norm_rope(q, k, w, w, 1e-6)
    for name, x in (("q", q), ("k", k)):
        check_rope(got[name], ref.norm_rope(x.double(), w, 1e-6, None, None), d, dtype)


# bf16 with rows enough for the kernel of 128 rows and row tiles too few for the machine, so that it splits keys: a
# chunk over long keys, a window far from sinks that end inside a tile, a batch whose sequences split and do not
# (tests/host/cache_plans_test.cpp holds the host layer to these plans; the shapes WAYS of test_gpu_cache_ops.py and its
# test of split keys leave such keys whole or take the kernel for few rows)
BIG_SPLIT = [((5000,), (200,), 1 << 20, 4, 4, 4), ((9000,), (150,), 6000, 70, 8, 4), ((7001, 90, 0, 5000), (130, 60, 0, 301), 1 << 40, 0, 4, 4),
             ((6000,), (513,), 2500, 33, 5, 2)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(BIG_SPLIT)))
def test_sink_attention_many_rows_split(case, d):
    import torch
    lens, nq, window, sink, G, H = BIG_SPLIT[case]
    g = gen(1100 + case)
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, sum(nq), H * G, d).transpose(0, 1)
    k, v = randn(g, H, sum(lens), d), randn(g, H, sum(lens), d)
    k = k + 2 * randn(g, H, 1, d)
    got = binding.sink_attention(q, k, v, window, sink, None, cu_q, cu_k, want_lse=True)
    for s, (m, n) in enumerate(zip(nq, lens)):
        if m == 0:
            continue
        rows = torch.tensor(sorted({0, m - 1, *(int(x) for x in np.linspace(0, m - 1, 23))}), device="cuda")
        seen = ref.seen_by(m, n, window, sink).cuda()[rows]
        a, x = int(cu_q[s]), int(cu_k[s])
        for h in sorted({0, G - 1, H * G - 1}):
            o, e, mass, size = ref.softmax_rows(q[h, a + rows].double(), k[h // G, x:x + n].double(),
                                                v[h // G, x:x + n].double(), seen, d ** -0.5)
            tol, tol_e = ref.attention_bounds(o, e, mass, size, n, d, True)
            assert bool(((got["out"][h, a + rows].double() - o).abs() <= tol).all()), (s, h)
            assert bool(((got["lse"][h, a + rows].double() - e).abs() <= tol_e).all()), (s, h)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_sink_attention_many_rows_split_unseen_values_do_not_matter(bad):
    import torch
    g = gen(1150)
    H, G, d, n, m, W, sink = 4, 4, 128, 6000, 200, 4000, 4
    q, k, v = randn(g, H * G, m, d), randn(g, H, n, d), randn(g, H, n, d)
    clean = binding.sink_attention(q, k, v, W, sink, None, [0, m], [0, n])["out"]
    seen = ref.seen_by(m, n, W, sink).cuda()
    for j in (2, 900, n - m - W + 1, n - m + 1, 3000, n - 1):
        v2 = v.clone()
        v2[:, j, 77] = bad
        got = binding.sink_attention(q, k, v2, W, sink, None, [0, m], [0, n])["out"]
        hit = torch.zeros((H * G, m, d), dtype=torch.bool, device="cuda")
        hit[:, seen[:, j], 77] = True
        assert torch.equal(got[~hit], clean[~hit]), j
        assert not bool(torch.isfinite(got[hit]).any()), j


# One token over many keys beside a prompt, whose work alone would leave its keys in one run; both orders.
LONE = [((1, 2048), (30000, 2048)), ((2048, 1), (2048, 30000)), ((3, 700, 0, 1500), (40000, 900, 5, 1500))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(LONE)))
def test_sink_attention_lone_sequence(case, dtype):
    import torch
    nq, lens = LONE[case]
    g = gen(1200 + case)
    H, G, d = 8, 4, 64
    cu_q, cu_k = cum(nq), cum(lens)
    q = randn(g, H * G, sum(nq), d, dtype=dtype)
    k, v = randn(g, H, sum(lens), d, dtype=dtype), randn(g, H, sum(lens), d, dtype=dtype)
    got = binding.sink_attention(q, k, v, 1 << 40, 0, None, cu_q, cu_k, want_lse=True)
    check_some_rows(got, q, k, v, cu_q, cu_k, d, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache4_attention_lone_sequence(dtype):
    import torch
    g = gen(1250)
    H, G, d, nq, rows = 4, 4, 64, (1, 6000), (40000, 6016)
    cache, kv = fill_cache(g, H, rows, d, dtype)
    cu_q, length = cum(nq), torch.tensor([rows] * H, dtype=torch.int32, device="cuda")
    q = randn(g, H * G, sum(nq), d, dtype=dtype)
    got = binding.cache4_attention(q, cache, length, None, cu_q, want_lse=True)
    check_some_rows(got, q, kv["keys"], kv["values"], cu_q, cache.cu_rows, d, dtype)


def check_some_rows(got, q, k, v, cu_q, cu_k, d, dtype):
    """Plain causal attention: the first and last rows of every sequence and a spread between, of three heads."""
    import torch
    G = q.shape[0] // k.shape[0]
    for s in range(len(cu_q) - 1):
        a, m, x, n = int(cu_q[s]), int(cu_q[s + 1] - cu_q[s]), int(cu_k[s]), int(cu_k[s + 1] - cu_k[s])
        if m == 0:
            continue
        rows = torch.tensor(sorted({0, m - 1, *(int(i) for i in np.linspace(0, m - 1, 9))}), device="cuda")
        seen = torch.arange(n, device="cuda")[None, :] <= (n - m + rows)[:, None]
        for h in (0, G + 1, q.shape[0] - 1):
            o, e, mass, size = ref.softmax_rows(q[h, a + rows].double(), k[h // G, x:x + n].double(),
                                                v[h // G, x:x + n].double(), seen, d ** -0.5)
            tol, tol_e = ref.attention_bounds(o, e, mass, size, n, d, dtype == "bf16")
            assert bool(((got["out"][h, a + rows].double() - o).abs() <= tol).all()), (s, h)
            assert bool(((got["lse"][h, a + rows].double() - e).abs() <= tol_e).all()), (s, h)
