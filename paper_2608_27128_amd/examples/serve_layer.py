"""One attention layer from prompt to decoding, with its cache evicted, repaired and held in 4 bits.

    python -m paper_2608_27128_amd.examples.serve_layer [--tokens 8192] [--seqs 2] [--steps 16]

The calls in the order a server makes them, on random projections (no model weights are needed):

1. ``qk_norm_rope``: the prompt's queries and keys, token major as projections leave them, normalised per
   head and rotated; the keys land head major, as the cache holds them.
2. ``sink_attention``: the prompt's attention under a streaming policy (a window and the first tokens).
3. ``select_topk`` and ``repair``: a policy's retained set, and the repaired one of the same budget.
4. ``cache4_compact``: the retained keys and values into a 4-bit cache with room for the answer.
5. per step ``qk_norm_rope``, ``cache4_append`` and ``cache4_attention`` for one new token per sequence.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from paper_2608_27128_amd import binding

N_SINK, EPS = 4, 1e-6


def rope_table(n_pos: int, d: int, theta: float = 1.0e6, device="cuda"):
    """cos of the d / 2 channel pairs, then sin, for every position: (n_pos, d) float32."""
    f = theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=device) / d)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


class Layer:
    """The state a server keeps for one layer: norm weights, the rotation's table, and the cache."""

    def __init__(self, lens, steps: int, n_heads: int = 8, group: int = 4, d: int = 128, budget_frac: float = 0.4,
                 window: int = 1024, dtype=torch.bfloat16):
        self.lens, self.steps, self.H, self.G, self.d, self.dtype = list(lens), steps, n_heads, group, d, dtype
        self.window, self.scale = window, d ** -0.5
        self.cu = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int64)
        self.one = np.arange(len(self.lens) + 1, dtype=np.int64)  # a token per sequence
        self.budget = np.array([max(1, int(budget_frac * n)) for n in self.lens], dtype=np.int64)
        self.q_weight, self.k_weight = torch.ones(d, device="cuda"), torch.ones(d, device="cuda")
        self.rope = rope_table(max(self.lens) + steps, d)
        self.positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in self.lens]).cuda()
        self.next = torch.tensor(self.lens, dtype=torch.int32, device="cuda")  # each sequence's next position
        self.cache = binding.Cache4.empty(n_heads, self.budget + steps, d)
        self.length = None

    def prompt(self, q, k, v, policy_scores, tau: float = 0.9, w: int = 32, n_recent: int = 64) -> dict:
        """Projections (T, heads, d) of all prompt tokens, and a policy's scores (n_heads, T): the attention's
        output, the repair's stats, and the filled cache."""
        r = binding.qk_norm_rope(q.transpose(0, 1), k.transpose(0, 1), self.q_weight, self.k_weight, EPS, self.rope,
                                 self.positions)
        v = v.transpose(0, 1)
        out = torch.empty_like(q)
        binding.sink_attention(r["q"], r["k"], v, self.window, N_SINK, self.scale, self.cu, self.cu,
                               out=out.transpose(0, 1))
        s0 = binding.select_topk(policy_scores, self.budget, N_SINK, n_recent, self.cu)["retained"]
        s1 = binding.repair(r["k"], s0, self.budget, tau, w, N_SINK, n_recent, self.cu, want_all=False)
        kept = binding.cache4_compact(r["k"], v, s1["s1"], self.cache, self.cu)
        self.length = kept["len"]
        return {"out": out, "keys": r["k"], "s1": s1["s1"], "repair": s1["stats"], "status": kept["status"]}

    def step(self, q, k, v) -> dict:
        """Projections (n_seqs, heads, d) of one new token per sequence: the attention's output over the
        cache, the new token included."""
        r = binding.qk_norm_rope(q.transpose(0, 1), k.transpose(0, 1), self.q_weight, self.k_weight, EPS, self.rope,
                                 self.next)
        grown = binding.cache4_append(r["k"], v.transpose(0, 1), self.cache, self.length, self.one, len_out=self.length)
        out = torch.empty_like(q)
        binding.cache4_attention(r["q"], self.cache, self.length, self.scale, self.one, out=out.transpose(0, 1))
        self.next += 1
        return {"out": out, "q": r["q"], "status": grown["status"]}


def projections(tokens: int, layer: Layer, gen):
    """Random q, k and v of so many tokens, as views of one token-major buffer; keys share a channel offset."""
    H, G = layer.H, layer.G
    x = torch.randn((tokens, H * G + 2 * H, layer.d), generator=gen, device="cuda")
    x[:, H * G:H * G + H] += 2.0 * torch.randn((1, H, layer.d), generator=gen, device="cuda")
    return x.to(layer.dtype).split([H * G, H, H], dim=1)


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=8192, help="of the longest prompt")
    ap.add_argument("--seqs", type=int, default=2)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    layer = Layer([max(1, a.tokens - 37 * s) for s in range(a.seqs)], a.steps)
    T = int(layer.cu[-1])
    # (random keys are far less alike than a model's: a threshold at which some are twins)
    got = layer.prompt(*projections(T, layer, gen), torch.rand((layer.H, T), generator=gen, device="cuda"), tau=0.55)
    orphans, donors, swaps, _ = got["repair"].sum(0).tolist()
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    tokens = [projections(a.seqs, layer, gen) for _ in range(a.steps)]
    start.record()
    for x in tokens:
        layer.step(*x)
    stop.record()
    torch.cuda.synchronize()
    held = sum(x.numel() for x in (layer.cache.k_codes, layer.cache.k_scales, layer.cache.v_codes, layer.cache.v_scales))
    print(f"prompts of {layer.lens} tokens: {orphans} orphans, {donors} donors, {swaps} swapped; "
          f"{held / 2**20:.1f} MiB of cache instead of {4 * T * layer.H * layer.d / 2**20:.1f}; "
          f"{1e3 * start.elapsed_time(stop) / a.steps:.0f} us a decode step; rows in use {layer.length[0].tolist()}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
