"""Edges of the operators around the cache on the GPU, against plain 64-bit forms (cache_ops_ref.py)."""
import math

import pytest

import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache_ops import check_rope, gen, randn

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
