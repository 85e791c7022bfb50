"""Accumulated attention weights where keys, queries or log-sum-exps are not finite: what exp(scale q . k - lse) is
there, for every kernel of them, and nothing of it in the sums of other keys."""
import math

import pytest

import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache8 import check_mass, lse_of
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


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_queries_without_weights_may_be_anything(shape, dtype, d):
    """Rows whose log-sum-exp is -inf, as the padding of a batch has it, weigh nothing whatever they hold; a
    log-sum-exp of +inf leaves finite scores no weight."""
    import torch
    n, nq, W, sink = SHAPES[shape]
    q, k, lse = inputs(10 + shape, n, nq, W, sink, dtype, d)
    old = torch.rand(k.shape[:2], generator=gen(shape), device="cuda")
    some = [(0, nq - 1), (2, nq // 2), (5, nq - 5), (6, nq - 3), (6, nq - 4)]
    padded = q.clone()
    for i, (h, t) in enumerate(some):
        lse[h, t] = -math.inf
        padded[h, t] = [math.nan, math.inf, -math.inf, math.nan, 1.0][i]
    padded[2, nq // 2, ::2] = -math.inf
    got = binding.attention_mass(padded, k, lse, W, sink, mass=old)["mass"]
    check_mass(got, q, k, lse, [0, nq], [0, n], lambda s, h, m, x: ref.seen_by(m, x, W, sink), d ** -0.5, old)
    clean = binding.attention_mass(q, k, lse, W, sink, mass=old)["mass"]
    for h, t in some:
        lse[h, t] = math.inf
    assert torch.equal(binding.attention_mass(q, k, lse, W, sink, mass=old)["mass"], clean)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_infinite_keys_and_queries_without_weights_together(dtype, d):
    """Both in one tile, beside a NaN query that has weights and spoils the keys that it sees, in a batch."""
    import torch
    H, G, lens = 2, 2, [700, 90]
    cu, T = [0, 700, 790], 790
    g = gen(77)
    q, k = randn(g, H * G, T, d, dtype=dtype), randn(g, H, T, d, dtype=dtype)
    q[:, :, 3] = 0.25 + q[:, :, 3].abs()
    lse = lse_of(q, k, cu, cu, T, 0, d ** -0.5)
    lse[0, 640] = lse[3, 780] = -math.inf
    clean = binding.attention_mass(q, k, lse, T, 0, None, cu, cu)["mass"]
    q[0, 640], q[3, 780], q[1, 300] = math.nan, math.inf, math.nan
    k[0, 500, 3] = k[1, 710, 3] = -math.inf
    got = binding.attention_mass(q, k, lse, T, 0, None, cu, cu)["mass"]
    assert bool(torch.isnan(got[0, :301]).all())
    assert float(got[0, 500]) == 0.0 and float(got[1, 710]) == 0.0
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[0, :301] = keep[0, 500] = keep[1, 710] = False
    # (sums that a row without weights touched may be computed in another way: 2^-24 a rounding, d + 8 of them a score of
    # at most 30, and one an addition of at most 1600)
    assert float((got[keep].double() - clean[keep].double()).abs().max()) <= \
        float(clean[keep].max()) * 2.0 ** -24 * 2 * ((d + 8) * 30 + 1600)
