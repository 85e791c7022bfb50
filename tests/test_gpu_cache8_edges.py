"""Edges of the accumulated weights and the 8-bit cache on the GPU: graphs, streams, offsets past 32 bits, strides,
scores that fill the LDS, values that are not finite, and a run of the calls together as a server makes them."""
import math

import numpy as np
import pytest

import cache8_ref as ref8
import cache_ops_ref as ref
from paper_2608_27128_amd import binding
from test_gpu_cache8 import check_mass, check_rows, filled, lse_of, poison
from test_gpu_cache_ops import check_attention, cum, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,nq,G", [(1000, 16, 1), (1024, 4, 4), (5000, 4, 4), (3000, 1, 16), (2100, 17, 1)])
def test_attention_scores_that_fill_the_lds(rows, nq, G, dtype):
    """16 rows a problem in one and in many splits, and one row more than a tile."""
    import torch
    g = gen(rows + nq)
    H, d = 2, 128
    cache, length, keys, values = filled(g, H, [rows], d, dtype)
    q = randn(g, H * G, nq, d, dtype=dtype)
    old = torch.rand(keys.shape[:2], generator=g, device="cuda")
    got = binding.cache8_attention(q, cache, length, None, [0, nq], want_lse=True, mass=old)
    for h in range(H):
        n = int(length[h, 0])
        seen = ref.seen_by(nq, n, 1 << 40, 0)
        hs = slice(h * G, h * G + G)
        check_attention(got["out"][hs][:1], q[hs][:1], keys[h:h + 1, :n], values[h:h + 1, :n], [0, nq], [0, n],
                        lambda *_: seen, d ** -0.5, dtype, got["lse"][hs][:1])
        check_mass(got["mass"][None, h, :n], q[hs], keys[h:h + 1, :n], got["lse"][hs], [0, nq], [0, n], lambda *_: seen,
                   d ** -0.5, old[None, h, :n])
        assert not bool(got["mass"][h, n:].any())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("sink", [1, 32, 33, 100, 300])
def test_mass_of_sinks_past_the_window(sink, dtype, d):
    """Sinks that many rows behind their window see: in one block of keys, in more, in all of a tile and the next; two
    sequences, the second with fewer keys than sinks, and old weights."""
    import torch
    g = gen(1000 + sink)
    H, G, W, cu = 2, 3, 100, [0, 1700, 1700 + 29]
    q, k = randn(g, H * G, cu[-1], d, dtype=dtype), randn(g, H, cu[-1], d, dtype=dtype)
    lse = lse_of(q, k, cu, cu, W, sink, d ** -0.5)
    old = torch.rand((H, cu[-1]), generator=g, device="cuda")
    got = binding.attention_mass(q, k, lse, W, sink, None, cu, cu, mass=old)["mass"]
    check_mass(got, q, k, lse, cu, cu, lambda s, h, m, n: ref.seen_by(m, n, W, sink), d ** -0.5, old)


@pytest.mark.parametrize("dtype,d,H,G", [("bf16", 128, 19, 1), ("bf16", 64, 8, 2), ("f32", 64, 9, 3), ("bf16", 128, 16, 1)])
def test_mass_of_many_heads(dtype, d, H, G):
    """Whole and partial groups of eight heads, ragged prompts whose rows are split."""
    g = gen(H + d)
    lens = [1300, 1, 400]
    cu = cum(lens)
    q, k = randn(g, H * G, sum(lens), d, dtype=dtype), randn(g, H, sum(lens), d, dtype=dtype)
    lse = lse_of(q, k, cu, cu, 2000, 0, 0.1)
    got = binding.attention_mass(q, k, lse, 2000, 0, 0.1, cu, cu)["mass"]
    check_mass(got, q, k, lse, cu, cu, lambda s, h, m, n: ref.seen_by(m, n, 2000, 0), 0.1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-90, -30, 30, 90])
def test_mass_of_fp32_at_every_magnitude(power, d):
    """Queries and keys scaled by powers of two that cancel weigh the same, bit for bit."""
    import torch
    g = gen(power + 200)
    H, G, n = 2, 2, 300
    q, k = randn(g, H * G, n, d, dtype="f32"), randn(g, H, n, d, dtype="f32")
    lse = lse_of(q, k, [0, n], [0, n], n, 0, 0.1)
    want = binding.attention_mass(q, k, lse, n, 0, 0.1)["mass"]
    got = binding.attention_mass(q * 2.0 ** power, k * 2.0 ** -power, lse, n, 0, 0.1)["mass"]
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [31, 512, 513, 2048, 2049, 4096, 4097, 16385, 32768, 32769, 50000])
def test_evict_selects_at_every_length(rows):
    """Lengths at and around those where the selection takes another number of threads, or does not keep its keys: the
    kept rows of two heads of their own lengths, weights with ties, and a problem beside them that has one row."""
    import torch
    g = gen(rows)
    H, d, budget = 2, 64, [rows // 2 + 1, 1]
    cache, to = binding.Cache8.empty(H, [rows, 1], d), binding.Cache8.empty(H, budget, d)
    for c in (cache.k_codes, cache.v_codes):
        c.zero_()
    for c in (cache.k_scales, cache.v_scales):
        c.fill_(127)
    r0 = int(cache.cu_rows[1])
    length = torch.tensor([[rows, 1], [rows - rows // 5, 0]], dtype=torch.int32, device="cuda")
    mass = (torch.rand((H, int(cache.cu_rows[-1])), generator=g, device="cuda") * 3000).floor() / 64
    got = binding.cache8_evict(cache, length, mass, budget, to, 4, 16)
    for h in range(H):
        n, m = int(length[h, 0]), int(got["len"][h, 0])
        kept = ref8.kept_rows(mass[h, :n].tolist(), n, budget[0], 4, 16)
        assert m == len(kept) and got["pos"][h, :m].tolist() == list(kept)
        assert bool((got["pos"][h, m:int(to.cu_rows[1])] == -1).all())
    assert got["len"][:, 1].tolist() == [1, 0]
    assert got["mass"][:, int(to.cu_rows[1])].tolist() == [float(mass[0, r0]), 0.0]


def test_evict_selects_of_many_long_problems():
    """More problems than CUs, the longest between 4096 and 8192 rows."""
    import torch
    g = gen(77)
    H, d, rows = 150, 64, [5000, 90]
    cache, to = binding.Cache8.empty(H, rows, d), binding.Cache8.empty(H, [64, 64], d)
    for c in (cache.k_codes, cache.v_codes):
        c.zero_()
    for c in (cache.k_scales, cache.v_scales):
        c.fill_(127)
    length = torch.tensor([rows] * H, dtype=torch.int32, device="cuda")
    length[:, 0] -= torch.arange(H, device="cuda", dtype=torch.int32)
    mass = (torch.rand((H, int(cache.cu_rows[-1])), generator=g, device="cuda") * 300).floor() / 64
    got = binding.cache8_evict(cache, length, mass, [50, 61], to, 4, 16)
    for h in range(0, H, 7):
        for s in range(2):
            n, r0, t0 = int(length[h, s]), int(cache.cu_rows[s]), int(to.cu_rows[s])
            kept = ref8.kept_rows(mass[h, r0:r0 + n].tolist(), n, [50, 61][s], 4, 16)
            assert got["pos"][h, t0:t0 + len(kept)].tolist() == list(kept)
    assert got["len"].tolist() == [[50, 61]] * H


def test_attention_more_queries_than_rows():
    """A problem with fewer rows than queries: the first queries see nothing, and neither do those of an empty one."""
    import torch
    g = gen(3)
    H, G, d, nq = 2, 2, 64, 6
    cache, length, keys, _ = filled(g, H, [40, 40], d, lens=[[3, 0], [6, 1]])
    q = randn(g, H * G, 2 * nq, d)
    got = binding.cache8_attention(q, cache, length, None, [0, nq, 2 * nq], want_lse=True, want_mass=True)
    for h in range(H):
        for s in range(2):
            n = int(length[h, s])
            for x in range(G):
                rows = slice(s * nq, s * nq + nq - n)
                assert not bool(got["out"][h * G + x, rows].any())
                assert bool((got["lse"][h * G + x, rows] == -math.inf).all())
            hs, r0 = slice(h * G, h * G + G), int(cache.cu_rows[s])
            check_mass(got["mass"][None, h, r0:r0 + n], q[hs, s * nq:(s + 1) * nq], keys[h:h + 1, r0:r0 + n],
                       got["lse"][hs, s * nq:(s + 1) * nq], [0, nq], [0, n], lambda *_: ref.seen_by(nq, n, 1 << 40, 0), d ** -0.5)
    assert bool(torch.isfinite(got["mass"]).all())


def test_attention_large_scores_and_not_finite_queries():
    """Scores of thousands; a NaN query spoils its own output and its problem's weights, and nothing else."""
    import torch
    g = gen(5)
    H, G, d = 2, 4, 64
    cache, length, keys, values = filled(g, H, [700, 90], d)
    q = 30 * randn(g, H * G, 2, d)
    clean = binding.cache8_attention(q, cache, length, 1.0, [0, 1, 2], want_lse=True, want_mass=True)
    for h in range(H):
        n = int(length[h, 0])
        seen = ref.seen_by(1, n, 1 << 40, 0)
        check_attention(clean["out"][h * G:h * G + 1, :1], q[h * G:h * G + 1, :1], keys[h:h + 1, :n], values[h:h + 1, :n],
                        [0, 1], [0, n], lambda *_: seen, 1.0, "bf16", clean["lse"][h * G:h * G + 1, :1])
    q2 = q.clone()
    q2[1, 0] = math.nan
    got = binding.cache8_attention(q2, cache, length, 1.0, [0, 1, 2], want_mass=True)
    assert bool(torch.isnan(got["out"][1, 0]).all()) and bool(torch.isnan(got["mass"][0, :int(length[0, 0])]).all())
    keep = torch.ones(H * G, 2, dtype=torch.bool, device="cuda")
    keep[1, 0] = False
    assert torch.equal(got["out"][keep], clean["out"][keep])
    assert torch.equal(got["mass"][1], clean["mass"][1]) and torch.equal(got["mass"][0, 704:], clean["mass"][0, 704:])


def test_offsets_past_32_bits():
    """A cache and keys of more than 4 GiB: the last head's results are those of that head alone."""
    import torch
    g = gen(7)
    H, d, n = 34, 128, 1 << 20
    small, length, _, _ = filled(g, 1, [n], d, lens=[[n - 5]])
    big = binding.Cache8.empty(H, n, d)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(big, name)[:-1] = 0 if "codes" in name else 100
        getattr(big, name)[-1] = getattr(small, name)[0]
    # (33 heads lie before the last: 33 * 2^27 bytes)
    lens = torch.full((H, 1), n - 5, dtype=torch.int32, device="cuda")
    q = randn(g, H * 2, 3, d)
    old = torch.rand((H, n), generator=g, device="cuda")
    a = binding.cache8_attention(q, big, lens, None, [0, 3], want_lse=True, mass=old)
    b = binding.cache8_attention(q[-2:], small, length, None, [0, 3], want_lse=True, mass=old[-1:].contiguous())
    # (splits differ with the number of heads: not the same bits)
    assert float((a["out"][-2:].float() - b["out"].float()).abs().max()) < 1e-3
    assert float((a["mass"][-1] - b["mass"][0]).abs().max()) < 1e-5
    to_a, to_b = binding.Cache8.empty(H, n // 2, d), binding.Cache8.empty(1, n // 2, d)
    ea = binding.cache8_evict(big, lens, old, n // 2, to_a)
    eb = binding.cache8_evict(small, length, old[-1:].contiguous(), n // 2, to_b)
    assert torch.equal(ea["pos"][-1], eb["pos"][0]) and torch.equal(to_a.v_codes[-1], to_b.v_codes[0])
    assert torch.equal(to_a.k_codes[-1], to_b.k_codes[0]) and torch.equal(to_a.k_scales[-1], to_b.k_scales[0])
    del big, to_a, ea
    # 17 heads of 2^20 keys of 256 bytes: the last begins past 2^32 bytes
    H, T = 17, 1 << 20
    k = torch.zeros((H, T, d), dtype=torch.bfloat16, device="cuda")
    k[-1] = randn(g, T, d)
    q = randn(g, H, 2, d)
    lse = lse_of(q[-1:], k[-1:], [0, 2], [0, T], T, 0, d ** -0.5).expand(H, 2).contiguous()
    a = binding.attention_mass(q, k, lse, T, 0)["mass"]
    b = binding.attention_mass(q[-1:], k[-1:], lse[-1:], T, 0)["mass"]
    assert torch.equal(a[-1], b[0]) and float(b.sum()) > 1.99


def test_strides_and_repeated_heads():
    """Token-major queries and keys, one KV head repeated (stride 0), rows that no 16 bytes divide (copied)."""
    import torch
    g = gen(9)
    T, H, G, d = 300, 3, 2, 128
    qkv = randn(g, T, H * G + H, d)
    q, k = (x.transpose(0, 1) for x in qkv.split([H * G, H], 1))
    lse = lse_of(q, k, [0, T], [0, T], 50, 4, d ** -0.5)
    want = binding.attention_mass(q.contiguous(), k.contiguous(), lse, 50, 4)["mass"]
    assert torch.equal(binding.attention_mass(q, k, lse, 50, 4)["mass"], want)
    wide = torch.zeros((H, T, d + 4), dtype=torch.bfloat16, device="cuda")
    wide[:, :, :d] = k
    assert torch.equal(binding.attention_mass(q, wide[:, :, :d], lse, 50, 4)["mass"], want)
    one = k[:1].expand(H, T, d)
    lse1 = lse_of(q, one, [0, T], [0, T], 50, 4, d ** -0.5)
    assert torch.equal(binding.attention_mass(q, one, lse1, 50, 4)["mass"],
                       binding.attention_mass(q, one.contiguous(), lse1, 50, 4)["mass"])
    cache = poison(binding.Cache8.empty(H, T, d))
    ones = torch.ones((H, T), dtype=torch.uint8, device="cuda")
    got = binding.cache8_compact(one, k, ones, cache)
    check_rows(cache, got["len"], [[[ref8.stored(k[0].double())[0], ref8.stored(k[h].double())[0]]] for h in range(H)],
               torch.bfloat16)


def step_calls(st):
    """A decode step and an eviction on fixed buffers; the cache grows by a row and is cut back."""
    n = binding.cache8_append(st["k"], st["v"], st["cache"], st["len"], st["one"], workspace=st["ws"])
    a = binding.cache8_attention(st["q"], st["cache"], n["len"], None, st["one"], want_lse=True, mass=st["mass"],
                                 workspace=st["ws"])
    e = binding.cache8_evict(st["cache"], n["len"], a["mass"], st["budget"], st["to"], 2, 8, workspace=st["ws"])
    r = binding.cache8_read(st["to"], e["len"], st["q"].dtype, workspace=st["ws"])
    m = binding.attention_mass(st["q"], st["raw"], a["lse"], 1 << 40, 0, None, st["one"], st["cu_raw"], workspace=st["ws"])
    return [n["len"], a["out"], a["lse"], a["mass"], e["len"], e["pos"], e["mass"], r["keys"], r["values"], m["mass"]]


def make_step(seed):
    import torch
    g = gen(seed)
    H, G, d, S = 2, 4, 128, 3
    st = {"one": cum([1] * S), "budget": [600, 20, 64], "cu_raw": cum([500, 700, 3])}
    st["cache"], st["len"], _, _ = filled(g, H, [900, 31, 96], d, lens=[[880, 31, 90], [900, 5, 64]])
    st["to"] = binding.Cache8.empty(H, st["budget"], d)
    st["k"], st["v"], st["q"] = randn(g, H, S, d), randn(g, H, S, d), randn(g, H * G, S, d)
    st["raw"] = randn(g, H, 1203, d)
    st["mass"] = torch.rand((H, int(st["cache"].cu_rows[-1])), generator=g, device="cuda")
    st["ws"] = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    return st


def test_graph_capture_and_replays():
    """The calls captured once and replayed with new inputs, eager work and synchronisations in between: every replay
    gives what the eager calls give."""
    import torch
    st = make_step(1)
    step_calls(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step_calls(st)
    for seed in (2, 3, 4):
        new = make_step(seed)
        for name in ("k", "v", "q", "raw", "mass", "len"):
            st[name].copy_(new[name])
        for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
            getattr(st["cache"], name).copy_(getattr(new["cache"], name))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        want = step_calls(new)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_two_graphs_with_workspaces_of_their_own():
    """Two captured steps replayed at once on two streams, each with its own workspace."""
    import torch
    sts = [make_step(5), make_step(6)]
    want = [[x.clone() for x in step_calls(make_step(s))] for s in (5, 6)]
    graphs, outs = [], []
    for st in sts:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step_calls(st))
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            for a, b in zip(x, y):
                assert torch.equal(a, b)


def test_another_stream():
    """Calls go to the current stream: behind work that is queued there."""
    import torch
    st, want = make_step(8), [x.clone() for x in step_calls(make_step(8))]
    q, late = st["q"].clone(), st["q"]
    late.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(20_000_000)
        late.copy_(q)
        got = step_calls(st)
        torch.cuda.current_stream().synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_poisoned_workspaces():
    """Results do not depend on what a workspace holds."""
    import torch
    st = make_step(9)
    want = None
    for fill in (0, 255, 127):
        new = make_step(9)
        new["ws"].fill_(fill)
        got = step_calls(new)
        want = want or got
        for x, y in zip(got, want):
            assert torch.equal(x, y)
    assert len(want) == 10 and st["ws"].numel() == 8 << 20
    # prompts, whose rows are split
    g = gen(10)
    q, k = randn(g, 8, 3000, 64), randn(g, 2, 3000, 64)
    lse = lse_of(q, k, [0, 3000], [0, 3000], 3000, 0, 0.125)
    first = None
    for fill in (0, 255):
        ws = torch.full((16 << 20,), fill, dtype=torch.uint8, device="cuda")
        got = binding.attention_mass(q, k, lse, 3000, 0, workspace=ws)["mass"]
        first = got if first is None else first
        assert torch.equal(got, first)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32")])
def test_a_layer_under_a_budget(d, dtype):
    """A prompt, its weights, the repaired set, and decoding with evictions in between: every call's result against the
    plain forms on what the call was given."""
    import torch
    from paper_2608_27128_amd.examples import evict_layer
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lens, steps, H, G = [300, 170], 14, 2, 4
    layer = evict_layer.Layer(lens, steps, n_heads=H, group=G, d=d, budget_frac=0.4, room=5, n_recent=8, dtype=dt)
    g = gen(12)
    got = layer.prompt(*evict_layer.projections(sum(lens), layer, g), tau=0.5)
    q, k, cu = got["q"], got["keys"], layer.cu
    lse = lse_of(q, k, cu, cu, 300, 0, layer.scale)
    tol = 1e-4 * got["mass"].abs() + 1e-5                        # (the calls took their own log-sum-exps)
    exact = torch.zeros_like(got["mass"], dtype=torch.float64)
    for s in range(2):
        a, b = int(cu[s]), int(cu[s + 1])
        for h in range(H):
            hs = slice(h * G, h * G + G)
            exact[h, a:b], _ = ref8.mass_of(q[hs, a:b].double(), k[h, a:b].double(), lse[hs, a:b].double(),
                                            ref.seen_by(b - a, b - a, 300, 0).cuda(), layer.scale)
    assert bool(((got["mass"].double() - exact).abs() <= tol).all())
    assert got["s1"].sum(1).tolist() == [int(layer.budget.sum())] * H
    evictions = 0
    for t in range(steps):
        n0, had = layer.length.clone(), layer.mass.clone()
        rows = binding.cache8_read(layer.cache, layer.length, torch.float32)
        x = evict_layer.projections(len(lens), layer, g)
        if layer.left == 0:
            kept = layer.evict()
            evictions += 1
            for h in range(H):
                for s in range(2):
                    r0 = int(layer.spare.cu_rows[s])
                    want = ref8.kept_rows(had[h, r0:r0 + int(n0[h, s])].tolist(), int(n0[h, s]), int(layer.budget[s]),
                                          evict_layer.N_SINK, layer.n_recent)
                    assert int(kept["len"][h, s]) == len(want) == int(layer.budget[s])
                    t0 = int(layer.cache.cu_rows[s])
                    now = binding.cache8_read(layer.cache, layer.length, torch.float32)
                    assert torch.equal(now["keys"][h, t0:t0 + len(want)].double(),
                                       ref8.stored(rows["keys"][h, r0 + torch.tensor(want, device="cuda")].double())[0])
        old = layer.mass.clone()
        res = layer.step(*x)
        assert not bool(res["status"].any())
        now = binding.cache8_read(layer.cache, layer.length, torch.float32)
        for s in range(2):
            for h in range(H):
                n, r0 = int(layer.length[h, s]), int(layer.cache.cu_rows[s])
                kk, vv, hs = now["keys"][h:h + 1, r0:r0 + n], now["values"][h:h + 1, r0:r0 + n], slice(h * G, h * G + G)
                seen = ref.seen_by(1, n, 1 << 40, 0)
                check_attention(res["out"][s:s + 1, hs].transpose(0, 1)[:1], res["q"][hs, s:s + 1][:1], kk, vv, [0, 1], [0, n],
                                lambda *_: seen, layer.scale, dtype)
                e = lse_of(res["q"][hs, s:s + 1], kk, [0, 1], [0, n], n, 0, layer.scale)
                w, off = ref8.mass_of(res["q"][hs, s:s + 1].double(), kk[0].double(), e.double(), seen.cuda(), layer.scale)
                err = (layer.mass[h, r0:r0 + n].double() - old[h, r0:r0 + n].double() - w).abs()
                assert bool((err <= 2 * off + 1e-5 * w + 2e-6 * (1 + old[h, r0:r0 + n].double())).all()), (t, h, s)
    assert evictions == 2 and layer.length[0].tolist() == [int(b) + 4 for b in layer.budget]


def test_the_example_runs():
    """The example's own run, with its printing."""
    import sys
    from paper_2608_27128_amd.examples import evict_layer
    argv, sys.argv = sys.argv, ["evict_layer", "--tokens", "700", "--steps", "70"]
    try:
        assert evict_layer.main() == 0
    finally:
        sys.argv = argv
