"""Accumulated attention weights where keys, queries or log-sum-exps are not finite: what exp(scale q . k - lse) is
there, for every kernel of them, and nothing of it in the sums of other keys."""
import math

import pytest

from paper_2608_27128_amd import binding
from test_gpu_cache8 import lse_of
from test_gpu_cache_ops import gen, randn

pytestmark = pytest.mark.gpu

# tokens, queries, window, sinks: whole prompts, split and not, a window, an observation window of few rows
SHAPES = [(1500, 1500, 1500, 0), (300, 300, 40, 3), (2000, 30, 2000, 0), (40, 900, 1 << 40, 0)]


def inputs(seed, n, nq, W, sink, dtype, d, H=2, G=4):
    g = gen(seed)
    q, k = randn(g, H * G, nq, d, dtype=dtype), randn(g, H, n, d, dtype=dtype)
    q[:, :, 3] = 0.25 + q[:, :, 3].abs()      # channels of one sign: an infinite key's scores have one too
    q[:, :, 7] = -0.25 - q[:, :, 7].abs()
    q[:, :, 11] = 0
    return q, k, lse_of(q, k, [0, nq], [0, n], W, sink, d ** -0.5)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_keys_with_infinite_elements(shape, dtype, d):
    """Scores of -inf weigh 0, of +inf infinitely much, and those that are no number make the sum none."""
    import torch
    n, nq, W, sink = SHAPES[shape]
    q, k, lse = inputs(shape, n, nq, W, sink, dtype, d)
    clean = binding.attention_mass(q, k, lse, W, sink)["mass"]
    bad = k.clone()
    want = {}
    for j, (parts, sums) in enumerate([({3: -math.inf}, 0.0), ({7: math.inf}, 0.0), ({3: math.inf}, math.inf),
                                       ({3: -math.inf, 7: math.inf}, 0.0), ({3: math.inf, 7: math.inf}, math.nan),
                                       ({11: math.inf}, math.nan), ({5: math.nan}, math.nan)]):
        at = n // 2 + 2 * j if n > 100 else 2 * j  # (a query sees each of them)
        want[at] = sums
        for c, x in parts.items():
            bad[1, at, c] = x
    got = binding.attention_mass(q, bad, lse, W, sink)["mass"]
    rest = torch.ones_like(clean, dtype=torch.bool)
    for at, sums in want.items():
        rest[1, at] = False
        x = float(got[1, at])
        assert (math.isnan(x) if math.isnan(sums) else x == sums), (at, sums, x)
    assert torch.equal(got[rest], clean[rest])
