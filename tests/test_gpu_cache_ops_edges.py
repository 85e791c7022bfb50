"""Edges of the operators around the cache on the GPU, against plain 64-bit forms (cache_ops_ref.py)."""
import pytest

from paper_2608_27128_amd import binding
from test_gpu_cache_ops import gen, randn

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
