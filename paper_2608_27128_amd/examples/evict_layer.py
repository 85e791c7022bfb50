"""One attention layer from prompt to decoding under a fixed budget: its cache is held in 8 bits, and what attention
gives each row decides which rows go when it is full.

    python -m paper_2608_27128_amd.examples.evict_layer [--tokens 4096] [--seqs 2] [--steps 200]

The calls in the order a server makes them, on random projections (no model weights are needed):

1. ``qk_norm_rope`` and ``sink_attention`` over the whole prompt, with the queries' log-sum-exps.
2. ``attention_mass``: the weight that every token has received, the policy's scores.
3. ``select_topk`` and ``repair``: the retained set of those scores, and the repaired one of the same budget.
4. ``cache8_compact``: the retained rows and their weights into an 8-bit cache with room for some more.
5. per step ``cache8_append`` and ``cache8_attention``, which adds the step's weights to the rows'; when the room is
   used up ``cache8_evict`` moves the rows of most weight, the first and the last, into the spare cache, and the two
   change places (a server has one spare for all of its layers).
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from paper_2608_27128_amd import binding
from paper_2608_27128_amd.examples.serve_layer import EPS, N_SINK, projections, rope_table


class Layer:
    """The state a server keeps for one layer: norm weights, the rotation's table, the cache and its spare."""

    def __init__(self, lens, steps: int, n_heads: int = 8, group: int = 4, d: int = 128, budget_frac: float = 0.25,
                 room: int = 64, n_recent: int = 32, dtype=torch.bfloat16):
        self.lens, self.H, self.G, self.d, self.dtype = list(lens), n_heads, group, d, dtype
        self.n_recent, self.scale = n_recent, d ** -0.5
        self.cu = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int64)
        self.one = np.arange(len(self.lens) + 1, dtype=np.int64)  # a token per sequence
        self.budget = np.array([max(1, int(budget_frac * n)) for n in self.lens], dtype=np.int64)
        self.room = room
        self.q_weight, self.k_weight = torch.ones(d, device="cuda"), torch.ones(d, device="cuda")
        self.rope = rope_table(max(self.lens) + steps, d)
        self.positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in self.lens]).cuda()
        self.next = torch.tensor(self.lens, dtype=torch.int32, device="cuda")  # each sequence's next position
        self.cache, self.spare = (binding.Cache8.empty(n_heads, self.budget + room, d) for _ in range(2))
        self.length = self.mass = self.pos = None
        self.left = room

    def prompt(self, q, k, v, tau: float = 0.9, w: int = 32) -> dict:
        """Projections (T, heads, d) of all prompt tokens: the attention's output, the tokens' weights, the repair's
        stats, and the filled cache."""
        r = binding.qk_norm_rope(q.transpose(0, 1), k.transpose(0, 1), self.q_weight, self.k_weight, EPS, self.rope,
                                 self.positions)
        v, window = v.transpose(0, 1), max(self.lens)
        out = torch.empty_like(q)
        got = binding.sink_attention(r["q"], r["k"], v, window, 0, self.scale, self.cu, self.cu, want_lse=True,
                                     out=out.transpose(0, 1))
        mass = binding.attention_mass(r["q"], r["k"], got["lse"], window, 0, self.scale, self.cu, self.cu)["mass"]
        s0 = binding.select_topk(mass, self.budget, N_SINK, self.n_recent, self.cu)["retained"]
        s1 = binding.repair(r["k"], s0, self.budget, tau, w, N_SINK, self.n_recent, self.cu, want_all=False)
        kept = binding.cache8_compact(r["k"], v, s1["s1"], self.cache, self.cu, token_mass=mass)
        self.length, self.mass, self.pos = kept["len"], kept["mass"], kept["pos"]
        return {"out": out, "q": r["q"], "keys": r["k"], "mass": mass, "s1": s1["s1"], "repair": s1["stats"],
                "status": kept["status"]}

    def step(self, q, k, v) -> dict:
        """Projections (n_seqs, heads, d) of one new token per sequence: the attention's output over the cache, the
        new token included."""
        if self.left == 0:
            self.evict()
        r = binding.qk_norm_rope(q.transpose(0, 1), k.transpose(0, 1), self.q_weight, self.k_weight, EPS, self.rope,
                                 self.next)
        grown = binding.cache8_append(r["k"], v.transpose(0, 1), self.cache, self.length, self.one, len_out=self.length)
        out = torch.empty_like(q)
        binding.cache8_attention(r["q"], self.cache, self.length, self.scale, self.one, mass=self.mass,
                                 mass_out=self.mass, out=out.transpose(0, 1))
        self.next += 1
        self.left -= 1
        return {"out": out, "q": r["q"], "keys": r["k"], "status": grown["status"]}

    def evict(self) -> dict:
        """Back to the budget; rows appended since the last time have no position of their own here (-1)."""
        got = binding.cache8_evict(self.cache, self.length, self.mass, self.budget, self.spare, N_SINK, self.n_recent,
                                   pos=self.pos)
        self.cache, self.spare = self.spare, self.cache
        self.length, self.mass, self.pos, self.left = got["len"], got["mass"], got["pos"], self.room
        return got


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096, help="of the longest prompt")
    ap.add_argument("--seqs", type=int, default=2)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    layer = Layer([max(1, a.tokens - 37 * s) for s in range(a.seqs)], a.steps)
    # (random keys are far less alike than a model's: a threshold at which some are twins)
    got = layer.prompt(*projections(int(layer.cu[-1]), layer, gen), tau=0.55)
    orphans, donors, swaps, _ = got["repair"].sum(0).tolist()
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    tokens = [projections(a.seqs, layer, gen) for _ in range(a.steps)]
    start.record()
    for x in tokens:
        layer.step(*x)
    stop.record()
    torch.cuda.synchronize()
    print(f"prompts of {layer.lens} tokens: {orphans} orphans, {donors} donors, {swaps} swapped; "
          f"{1e3 * start.elapsed_time(stop) / a.steps:.0f} us a decode step; rows in use {layer.length[0].tolist()}, "
          f"budget {layer.budget.tolist()}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
