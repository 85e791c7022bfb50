"""Eviction by accumulated attention weight and the 8-bit cache that it is applied to, as cases that can be
timed and compared: the weight that every cached token has received, a cache in 8 bits with one scale for 32
tokens of a head, attention over that cache, and the eviction of the rows that received least.

Kinds:
  mass      the softmax weight that each key receives from the queries, summed over them and over the query
            heads that share the key; the queries' log-sum-exp is at hand from their attention
  compact8  the retained keys and values (and their weights) gathered into an 8-bit cache, and read back
  attn8     attention of a few query tokens over an 8-bit cache, with or without the rows' weights
  step8     one layer's decode step: the new token into the cache, attention, and the rows' weights
  evict8    the rows of most weight, the first and the last, moved into another cache, and read back

Shapes are those of the repository's workloads (8 KV heads a layer, 36x8 heads for whole models, d 128 and
64, 512 to 128k tokens, 64 ragged prompts), with 4 query heads to a KV head.

An 8-bit cache holds whole numbers of -127 .. 127 and, per head and 32 rows, one scale 2^(byte - 127) for the
keys and one for the values, the smallest with which every element rounds to 127 at most:
  k_codes  (H, C, d) int8
  k_scales (H, C/32) uint8
  v_codes  (H, C/8, d, 8) int8   blocks of 8 rows
  v_scales (H, C/32) uint8
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 32  # rows that share a scale


def _case(name, kind, **kw):
    c = {"kind": kind, "heads": 8, "group": 4, "seqs": 1, "lo": 1, "hi": 1, "d": 128, "dtype": "bf16",
         "nq": 1, "window": 0, "sink": 0, "frac": 0.5, "mass": False, "token_major": True, "len_seed": 0}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # every query of a 32k prompt, full causal attention: the largest work listed
        _case("mass_prompt_32k", "mass", lo=32768, hi=32768, nq=0, window=32768),
        # the same at d 64 and 8k tokens
        _case("mass_prompt_8k_d64", "mass", lo=8192, hi=8192, nq=0, window=8192, d=64),
        # the last 32 queries of 64 ragged prompts: an observation window
        _case("mass_last_32_64x", "mass", seqs=64, lo=1024, hi=4096, nq=32, window=4096),
        # fp32, ragged prompts in one batch, the streaming policy's window
        _case("mass_f32_ragged", "mass", group=1, seqs=5, lo=150, hi=1500, nq=0, d=64, dtype="f32", window=128, sink=4),
        # one layer's cache of an odd length, fp32, d 64
        _case("compact8_layer_4k", "compact8", lo=4001, hi=4001, d=64, dtype="f32", mass=True),
        # a whole 36-layer model's cache
        _case("compact8_36x8x16k", "compact8", heads=288, lo=16384, hi=16384, frac=0.4),
        # one layer at 128k cached rows, a few speculative tokens
        _case("attn8_layer_128k", "attn8", lo=131072, hi=131072, nq=4),
        # fp32 queries, d 64, ragged, weights wanted
        _case("attn8_f32_d64", "attn8", seqs=16, lo=500, hi=5000, nq=3, d=64, dtype="f32", mass=True),
        # the smallest decode step: one sequence, one layer, a cache of 512 rows
        _case("step8_512", "step8", lo=512, hi=512, mass=True),
        # a decode step of 64 ragged sequences
        _case("step8_64x", "step8", seqs=64, lo=1024, hi=4096, mass=True),
        # one layer's cache cut back by the slack it has grown
        _case("evict8_layer_4k", "evict8", lo=4224, hi=4224, frac=0.97),
        # 64 ragged sequences cut to three quarters
        _case("evict8_64x", "evict8", seqs=64, lo=1024, hi=4096, frac=0.75),
    ]


def _lens(case):
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    g = np.random.Generator(np.random.PCG64(np.random.SeedSequence(case["len_seed"], spawn_key=(n, lo, hi))))
    return [int(x) for x in g.integers(lo, hi + 1, size=n)]


def _queries(case, lens):
    """Query tokens of each sequence: nq of them at its end, or (nq = 0) all of its tokens."""
    return [min(n, case["nq"]) if case["nq"] else n for n in lens]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    """A case of the same ranges: prompts and caches from a few tokens to 128k, one sequence or a ragged batch,
    both head sizes and types, 1 to 8 query heads a KV head, one to 512 query tokens or the whole prompt."""
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["mass", "mass", "compact8", "attn8", "step8", "evict8"])
        seqs = rng.choice([1, 1, 2, 5, 16, 64])
        longest = {"mass": 32768, "compact8": 32768, "attn8": 131072, "step8": 131072, "evict8": 32768}[kind]
        hi = _log(rng, 16, longest)
        lo = hi if seqs == 1 else max(1, int(hi * rng.choice([0.05, 0.25, 0.7])))
        heads = rng.choice([1, 8, 8, 40, 288]) if kind in ("compact8", "evict8") else rng.choice([2, 8, 8, 8])
        nq = {"mass": rng.choice([0, 0, 1, _log(rng, 2, 512)]), "attn8": rng.choice([1, 1, 2, 7])}.get(kind, 1)
        window = rng.choice([hi, hi, _log(rng, 16, hi) if hi > 16 else hi])
        c = _case(None, kind, heads=heads, group=rng.choice([1, 2, 4, 4, 8]), seqs=seqs, lo=lo, hi=hi,
                  d=rng.choice([64, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), nq=nq, window=window,
                  sink=rng.choice([0, 4, 16]), frac=rng.choice([0.1, 0.3, 0.5, 0.75, 0.97]),
                  mass=rng.choice([True, False]), token_major=rng.choice([True, True, False]),
                  len_seed=rng.randrange(1 << 20))
        elements = heads * (c["group"] if kind == "mass" else 1) * seqs * hi * c["d"]
        if _cost(c) * (8 if c["dtype"] == "f32" else 1) <= 0.5 * top and elements <= 1.2e9:
            return c


# ---------------------------------------------------------------- the 8-bit format, plainly

def _blocks_of(x):
    """(H, C, d) as (H, C/32, 32 d)."""
    return x.reshape(x.shape[0], x.shape[1] // BLOCK, -1)


def _byte(amax):
    """The scale's byte for the largest magnitude of a block (fp32)."""
    return (((amax.view(torch.int32) + 0x10000) >> 23) - 6).clamp(1, 248)


def _power(e):
    """2^e, e an integer tensor in [-126, 127]."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes (int8, x's shape) and scale bytes (uint8, one per 32 rows) of (H, C, d) fp32 rows, C a multiple of 32."""
    b = _blocks_of(x)
    byte = _byte(b.abs().amax(dim=-1, keepdim=True))
    return torch.round(b * _power(127 - byte)).to(torch.int8).reshape(x.shape), byte.squeeze(-1).to(torch.uint8)


def _values(code, byte):
    """What codes (H, C, d) under scale bytes (H, C/32) stand for, in fp32."""
    return (_blocks_of(code).float() * _power(byte.int() - 127).unsqueeze(-1)).reshape(code.shape)


def _pack(kc, kb, vc, vb):
    """The cache's arrays from codes (H, C, d) and scale bytes (H, C/32) of keys and values."""
    H, C, d = kc.shape
    return {"k_codes": kc.contiguous(), "k_scales": kb.contiguous(),
            "v_codes": vc.reshape(H, C // 8, 8, d).transpose(2, 3).contiguous(), "v_scales": vb.contiguous()}


def _unpack(c):
    """Codes (H, C, d) and scale bytes of the keys and of the values."""
    H, C, d = c["k_codes"].shape
    return (c["k_codes"], c["k_scales"]), (c["v_codes"].transpose(2, 3).reshape(H, C, d), c["v_scales"])


# ---------------------------------------------------------------- inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(case, g, H, T):
    """Keys with a channel offset of their head, as the repository's synthetic caches have them."""
    return (_randn(g, H, T, case["d"]) + 2.0 * _randn(g, H, 1, case["d"])).to(_dtype(case))


def _heads_of(case, g, H, T):
    """(H, T, d) projections, a view of a token-major buffer where the case says so."""
    if case["token_major"]:
        return _randn(g, T, H, case["d"]).to(_dtype(case)).transpose(0, 1)
    return _randn(g, H, T, case["d"]).to(_dtype(case))


def _cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int64)


def _budgets(case, lens):
    return [max(1, int(case["frac"] * n)) for n in lens]


def _reserve(H, cu_rows, d):
    """The arrays of a cache, as a program reserves them once."""
    C = int(cu_rows[-1])
    return {"k_codes": torch.zeros((H, C, d), dtype=torch.int8, device="cuda"),
            "k_scales": torch.zeros((H, C // BLOCK), dtype=torch.uint8, device="cuda"),
            "v_codes": torch.zeros((H, C // 8, d, 8), dtype=torch.int8, device="cuda"),
            "v_scales": torch.zeros((H, C // BLOCK), dtype=torch.uint8, device="cuda")}


def _weights(g, H, T):
    """Weights as attention leaves them: most small, a few large, and tokens that received none."""
    w = torch.rand((H, T), generator=g, device="cuda") ** 8 * 50.0
    return torch.where(w < 1e-6, 0.0, w)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    lens, H, G, d, kind, dt = _lens(case), case["heads"], case["group"], case["d"], case["kind"], _dtype(case)
    st = {"case": case, "lens": lens, "scale": d ** -0.5}
    if kind == "mass":
        nq, T = _queries(case, lens), sum(lens)
        st["nq"], st["cu_q"], st["cu_k"] = nq, _cum(nq), _cum(lens)
        st["q"], st["k"] = _heads_of(case, g, H * G, sum(nq)), _keys(case, g, H, T)
        st["lse"] = torch.empty((H * G, sum(nq)), dtype=torch.float32, device="cuda")
        for q0, q1, s, seen, _ in _scores(st, st["q"], st["k"]):
            st["lse"][:, q0:q1] = torch.logsumexp(s.masked_fill_(~seen, -math.inf), dim=-1).reshape(H * G, q1 - q0)
    if kind == "compact8":
        T, st["cu"], budget = sum(lens), _cum(lens), _budgets(case, lens)
        st["keys"], st["values"] = _keys(case, g, H, T), _randn(g, H, T, d).to(dt)
        score, st["retained"] = torch.rand((H, T), generator=g, device="cuda"), torch.zeros((H, T), dtype=torch.uint8, device="cuda")
        for a, n, b in zip(st["cu"], lens, budget):
            st["retained"][:, a:a + n].scatter_(1, score[:, a:a + n].topk(b, dim=1).indices, 1)
        st["cu_rows"] = _cum([(b + 31) // 32 * 32 for b in budget])
        st["cache"] = _reserve(H, st["cu_rows"], d)
        st["mass"] = _weights(g, H, T) if case["mass"] else None
    if kind in ("attn8", "step8", "evict8"):
        st["cu_rows"] = _cum([(n + case["nq"] + 31) // 32 * 32 for n in lens])
        C = int(st["cu_rows"][-1])
        packed = [_quantise(x) for x in (_keys(case, g, H, C).float(), _randn(g, H, C, d).to(dt).float())]
        st["cache"] = _pack(*packed[0], *packed[1])
        # heads of one layer keep the same number of rows, or a few less
        less = torch.randint(0, 9, (H, len(lens)), generator=g, device="cuda", dtype=torch.int32)
        st["len"] = (torch.tensor(lens, dtype=torch.int32, device="cuda") - less).clamp(min=1)
        st["mass"] = _weights(g, H, C) if case["mass"] or kind == "evict8" else None
    if kind == "attn8":
        st["cu_q"] = np.arange(len(lens) + 1, dtype=np.int64) * case["nq"]
        st["q"] = _heads_of(case, g, H * G, len(lens) * case["nq"])
    if kind == "step8":
        st["cu_q"] = np.arange(len(lens) + 1, dtype=np.int64)
        st["q"], st["keys"] = _heads_of(case, g, H * G, len(lens)), _keys(case, g, H, len(lens))
        st["values"] = _heads_of(case, g, H, len(lens))
        st["open"], st["cu_open"] = st["len"] // BLOCK * BLOCK, np.arange(len(lens) + 1, dtype=np.int64) * BLOCK
    if kind == "evict8":
        st["budget"] = np.array(_budgets(case, lens), dtype=np.int64)
        st["cu_to"] = _cum([(b + 31) // 32 * 32 for b in st["budget"]])
        st["to"] = _reserve(H, st["cu_to"], d)
        st["pos"] = torch.randint(1, 4, (H, C), generator=g, device="cuda").cumsum(dim=1).to(torch.int32)
    return st


# ---------------------------------------------------------------- the plain forms

def _scores(st, q, k):
    """Blocks of queries of every sequence over the keys that they can see: the queries' range among all, their
    scores (H, G, rows, cols), which of them are seen (rows, cols), and the keys' places among all."""
    c, dev = st["case"], q.device
    H, G, W, sink = c["heads"], c["group"], c["window"], c["sink"]
    for s, (n, m) in enumerate(zip(st["lens"], st["nq"])):
        k0, q0 = int(st["cu_k"][s]), int(st["cu_q"][s])
        step = max(1, min(1024, 2 ** 28 // (H * G * min(n, W + sink + 1024))))
        for a in range(0, m, step):
            b = min(m, a + step)
            p = torch.arange(n - m + a, n - m + b, device=dev)[:, None]
            lo = max(0, n - m + a - W + 1)
            j = torch.cat([torch.arange(min(sink, lo), device=dev), torch.arange(lo, n - m + b, device=dev)])
            far = p - j
            seen = (far >= 0) & ((far < W) | (j < sink))
            qq = q[:, q0 + a:q0 + b].reshape(H, G * (b - a), -1).float()
            kk = k[:, k0 + j].float().transpose(1, 2).contiguous()
            yield q0 + a, q0 + b, (torch.matmul(qq, kk) * st["scale"]).reshape(H, G, b - a, -1), seen, k0 + j


def _plain_mass(st):
    c = st["case"]
    H, G = c["heads"], c["group"]
    mass = torch.zeros((H, int(st["cu_k"][-1])), dtype=torch.float64, device="cuda")
    for q0, q1, s, seen, at in _scores(st, st["q"], st["k"]):
        w = torch.exp(s.sub_(st["lse"][:, q0:q1].reshape(H, G, q1 - q0, 1)))
        mass[:, at] += torch.where(seen, w, 0.0).sum(dim=2).double().sum(dim=1)
    return {"mass": mass.float()}


def _plain_compact8(st):
    c, lens, dev = st["case"], st["lens"], "cuda"
    H, C, dt = c["heads"], int(st["cu_rows"][-1]), _dtype(c)
    seq = torch.repeat_interleave(torch.arange(len(lens), device=dev), torch.tensor(lens, device=dev))
    start, row0 = torch.tensor(st["cu"][:-1], device=dev), torch.tensor(st["cu_rows"][:-1], device=dev)
    keep = st["retained"] != 0
    upto = torch.cat([torch.zeros((H, 1), dtype=torch.int64, device=dev), keep.cumsum(dim=1)], dim=1)
    length = upto[:, torch.tensor(st["cu"][1:], device=dev)] - upto[:, start]
    h, t = keep.nonzero(as_tuple=True)
    row = row0[seq[t]] + upto[h, t] - upto[h, start[seq[t]]]
    pos = torch.full((H, C), -1, dtype=torch.int32, device=dev)
    pos[h, row] = (t - start[seq[t]]).to(torch.int32)
    out = {"len": length.to(torch.int32), "pos": pos}
    for name in ("keys", "values"):
        x = torch.zeros((H, C, c["d"]), dtype=torch.float32, device=dev)
        x[h, row] = st[name][h, t].float()
        out[name] = _values(*_quantise(x)).to(dt)
    if st["mass"] is not None:
        out["mass"] = torch.zeros((H, C), dtype=torch.float32, device=dev)
        out["mass"][h, row] = st["mass"][h, t]
    return out


def _plain_attn8(st, keys, values, length, nq):
    """q (H*G, S*nq, d) over keys and values (H, C, d) in fp32; length (H, S) counts the rows."""
    q, cu_rows, mass = st["q"], st["cu_rows"], st["mass"]
    H, C, d = keys.shape
    S, dev = len(cu_rows) - 1, "cuda"
    G, top = q.shape[0] // H, int((cu_rows[1:] - cu_rows[:-1]).max())
    j = torch.arange(top, device=dev)
    at = (torch.tensor(cu_rows[:-1], device=dev)[:, None] + j).clamp(max=C - 1)
    i = torch.arange(nq, device=dev)
    seen = (j < (length[:, :, None, None] - (nq - 1 - i)[:, None]))[:, :, None].expand(H, S, G, nq, top)
    qq = q.float().reshape(H, G, S, nq, d).transpose(1, 2).reshape(H, S, G * nq, d)
    kk = keys[:, at.reshape(-1)].reshape(H, S, top, d).transpose(2, 3).contiguous()
    s = torch.where(seen.reshape(H, S, G * nq, top), torch.matmul(qq, kk) * st["scale"], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    l = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(l > 0, l, 1.0)
    o = torch.matmul(p, values[:, at.reshape(-1)].reshape(H, S, top, d))
    got = {"out": o.reshape(H, S, G, nq, d).transpose(1, 2).reshape(H * G, S * nq, d).to(q.dtype),
           "lse": (torch.log(l) + m).reshape(H, S, G, nq).transpose(1, 2).reshape(H * G, S * nq)}
    if mass is not None:
        got["mass"] = torch.zeros((H, C), dtype=torch.float32, device=dev)
        more = p.sum(dim=2, dtype=torch.float64)
        for x in range(S):
            a, b = int(cu_rows[x]), int(cu_rows[x + 1])
            use = torch.arange(b - a, device=dev) < length[:, x, None]
            got["mass"][:, a:b] = torch.where(use, mass[:, a:b].double() + more[:, x, :b - a], 0.0).float()
    return got


def _plain_append(st):
    """Codes and bytes of keys and values with one more row in every problem; the rows beside it in its block are
    rounded again where the block's scale has to grow."""
    h = torch.arange(st["case"]["heads"], device="cuda")[:, None]
    row = torch.tensor(st["cu_rows"][:-1], device="cuda") + st["len"]
    blk, rest = row // BLOCK, st["len"] % BLOCK
    out = []
    for (code, byte), new in zip(_unpack(st["cache"]), (st["keys"].float(), st["values"].float())):
        had = torch.where(rest > 0, byte[h, blk].int(), 1)
        want = torch.maximum(had, _byte(new.abs().amax(dim=-1)))
        code, byte = code.clone(), byte.clone()
        at = (blk * BLOCK)[:, :, None] + torch.arange(BLOCK, device="cuda")      # (H, S, 32) rows
        hh = h[:, :, None]
        code[hh, at] = torch.round(code[hh, at].float() * _power(had - want)[:, :, None, None]).to(torch.int8)
        code[h, row] = torch.round(new * _power(127 - want)[:, :, None]).to(torch.int8)
        byte[h, blk] = want.to(torch.uint8)
        out.append((code, byte))
    return out


def _plain_step8(st):
    (kc, kb), (vc, vb) = _plain_append(st)
    length = st["len"] + 1
    keys, values = _values(kc, kb), _values(vc, vb)
    got = _plain_attn8(st, keys, values, length, 1)
    h = torch.arange(st["case"]["heads"], device="cuda")[:, None, None]
    r = st["open"][:, :, None] + torch.arange(BLOCK, device="cuda")
    at, use = torch.tensor(st["cu_rows"][:-1], device="cuda")[:, None] + r, (r < length[:, :, None])[..., None]
    for name, x in (("keys", keys), ("values", values)):
        got[name] = torch.where(use, x[h, at], 0.0).reshape(kc.shape[0], -1, kc.shape[2]).to(_dtype(st["case"]))
    return dict(got, len=length)


def _kept_rows(st, h, s):
    """The rows of one problem that an eviction keeps, ascending: the first and last ones, then those of most weight
    (the lower row first where weights are equal)."""
    n, r0, budget = int(st["len"][h, s]), int(st["cu_rows"][s]), int(st["budget"][s])
    rank = st["mass"][h, r0:r0 + n].clone()
    rank[:st["case"]["sink"]] = math.inf
    rank[max(0, n - 64):] = math.inf
    return torch.sort(torch.sort(rank, descending=True, stable=True).indices[:budget]).values


def _plain_evict8(st):
    c, dev = st["case"], "cuda"
    H, S, C, C2 = c["heads"], len(st["lens"]), int(st["cu_rows"][-1]), int(st["cu_to"][-1])
    # every problem's rows ranked in one stable sort, by weight and then by problem
    n, cu, cu_to = st["len"], torch.tensor(st["cu_rows"], device=dev), torch.tensor(st["cu_to"], device=dev)
    seq = torch.repeat_interleave(torch.arange(S, device=dev), cu[1:] - cu[:-1])
    r = torch.arange(C, device=dev) - cu[seq]
    nn = n[:, seq]
    rank = torch.where((r < c["sink"]) | (r >= nn - 64), math.inf, st["mass"])
    rank = torch.where(r < nn, rank, -1.0)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    order = order.gather(1, torch.sort(seq[order], dim=1, stable=True).indices)
    place = torch.empty_like(order).scatter_(1, order, torch.arange(C, device=dev).expand(H, C)) - cu[seq]
    keep = (place < torch.minimum(torch.tensor(st["budget"], device=dev)[seq], nn))
    upto = torch.cat([torch.zeros((H, 1), dtype=torch.int64, device=dev), keep.cumsum(dim=1)], dim=1)
    h, t = keep.nonzero(as_tuple=True)
    row = cu_to[seq[t]] + upto[h, t] - upto[h, cu[seq[t]]]
    got = {"len": (upto[:, cu[1:]] - upto[:, cu[:-1]]).to(torch.int32)}
    got["pos"] = torch.full((H, C2), -1, dtype=torch.int32, device=dev)
    got["pos"][h, row] = st["pos"][h, t]
    got["mass"] = torch.zeros((H, C2), dtype=torch.float32, device=dev)
    got["mass"][h, row] = st["mass"][h, t]
    for name, (code, byte) in zip(("keys", "values"), _unpack(st["cache"])):
        x = torch.zeros((H, C2, c["d"]), dtype=torch.float32, device=dev)
        x[h, row] = code[h, t].float() * _power(byte[h, t // BLOCK].int() - 127)[:, None]
        got[name] = _values(*_quantise(x)).to(_dtype(c))
    return got


def _plain(st):
    kind = st["case"]["kind"]
    if kind == "mass":
        return _plain_mass(st)
    if kind == "compact8":
        return _plain_compact8(st)
    if kind == "attn8":
        keys, values = (_values(*x) for x in _unpack(st["cache"]))
        return _plain_attn8(st, keys, values, st["len"], st["case"]["nq"])
    return _plain_step8(st) if kind == "step8" else _plain_evict8(st)


# ---------------------------------------------------------------- the framework's calls

def _framework(st):
    from paper_2608_27128_amd import binding

    c = st["case"]
    kind, dt = c["kind"], _dtype(c)
    if kind == "mass":
        return binding.attention_mass(st["q"], st["k"], st["lse"], c["window"], c["sink"], st["scale"], st["cu_q"],
                                      st["cu_k"])
    cache = binding.Cache8(cu_rows=st["cu_rows"], **st["cache"])
    if kind == "compact8":
        got = binding.cache8_compact(st["keys"], st["values"], st["retained"], cache, st["cu"], token_mass=st["mass"])
        kv = binding.cache8_read(cache, got["len"], dt)
        out = {"len": got["len"], "pos": got["pos"], "keys": kv["keys"], "values": kv["values"]}
        return dict(out, mass=got["mass"]) if st["mass"] is not None else out
    if kind == "attn8":
        return binding.cache8_attention(st["q"], cache, st["len"], st["scale"], st["cu_q"], want_lse=True,
                                        want_mass=st["mass"] is not None, mass=st["mass"])
    if kind == "step8":
        grown = binding.cache8_append(st["keys"], st["values"], cache, st["len"], st["cu_q"])
        got = binding.cache8_attention(st["q"], cache, grown["len"], st["scale"], st["cu_q"], want_lse=True,
                                       want_mass=st["mass"] is not None, mass=st["mass"])
        return dict(got, len=grown["len"], **binding.cache8_read(cache, grown["len"], dt, first=st["open"],
                                                                 cu_out=st["cu_open"]))
    to = binding.Cache8(cu_rows=st["cu_to"], **st["to"])
    got = binding.cache8_evict(cache, st["len"], st["mass"], st["budget"], to, c["sink"], 64, pos=st["pos"])
    return dict(got, **binding.cache8_read(to, got["len"], dt))


def run(st):
    return _framework(st) if own else _plain(st)


# ---------------------------------------------------------------- what a pass cannot do without

def _visible(case):
    """Pairs of a query token and a key that it sees, and keys that any query sees, over all sequences."""
    pairs = keys = 0
    for n, m in zip(_lens(case), _queries(case, _lens(case))):
        p = np.arange(n - m, n, dtype=np.float64)
        first = np.minimum(p + 1, case["sink"])
        pairs += float((first + np.minimum(case["window"], p + 1 - first)).sum())
        keys += min(n, case["sink"] + case["window"] + m - 1)
    return pairs, keys


def work(case):
    H, G, d, kind, lens = case["heads"], case["group"], case["d"], case["kind"], _lens(case)
    e = 4.0 if case["dtype"] == "f32" else 2.0
    T, S = float(sum(lens)), float(len(lens))
    if kind == "mass":
        pairs, keys = _visible(case)
        n = float(sum(_queries(case, lens)))
        return {"bytes": H * (G * n * (d * e + 4.0) + keys * d * e + 4.0 * T), "flops": 2.0 * d * pairs * H * G}
    row = 2.0 * (d + 1.0 / BLOCK)                     # a cached key and value, in bytes
    if kind in ("compact8", "evict8"):
        kept = float(H * sum(_budgets(case, lens)))
        back = kept * (row + 2.0 * d * e)             # read back
        if kind == "compact8":
            more = 8.0 if case["mass"] else 0.0
            return {"bytes": kept * (2.0 * d * e + row + 4.0 + more) + back + H * T, "flops": kept * d * 8.0}
        return {"bytes": kept * (2.0 * row + 12.0) + 4.0 * H * T + back, "flops": kept * d * 8.0}
    n = case["nq"] * S
    got = {"bytes": H * (T * row + 2.0 * G * n * d * e + 4.0 * G * n), "flops": 4.0 * d * T * H * G * case["nq"]}
    if case["mass"]:
        got["bytes"] += 8.0 * H * T
    if kind == "step8":
        got["bytes"] += H * S * (2.0 * d * e + row + BLOCK * (row + 2.0 * d * e))
    return got


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_8bit(x):
    """The values that (n, d) 64-bit rows have as the first of a problem's cache: 32 rows at a time, on the
    coarsest grid of the type that every one of them needs, ties to the even number."""
    n, d = x.shape
    b = torch.cat([x, x.new_zeros((-n % BLOCK, d))]).reshape(-1, BLOCK * d)
    frac, power = torch.frexp(b.abs().amax(dim=1, keepdim=True))
    e = torch.where(frac > 0, power - 7 + (frac >= 127.5 / 128).int(), -126).clamp(min=-126).long()
    grid = ((e + 1023) << 52).view(torch.float64)                 # 2^e
    return (torch.round(b / grid) * grid).reshape(-1, d)[:n]


def _exact_rows(cache):
    """The cached keys and values in 64 bits: whole numbers times powers of two."""
    H, C, d = cache["k_codes"].shape
    k, v = cache["k_codes"].double(), cache["v_codes"].double().permute(0, 1, 3, 2).reshape(H, C, d)
    return [x * ((b.long() + 896) << 52).view(torch.float64).repeat_interleave(BLOCK, dim=1)[:, :, None]
            for x, b in ((k, cache["k_scales"]), (v, cache["v_scales"]))]


def _exact_attn8(st, keys, values, count, nq):
    q, cu_rows = st["q"], st["cu_rows"]
    H, C = keys.shape[:2]
    G = q.shape[0] // H
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    mass = torch.zeros((H, C), dtype=torch.float64, device="cuda")
    for h in range(H):
        for s in range(len(cu_rows) - 1):
            r0, n = int(cu_rows[s]), count[h][s]
            x = q[h * G:h * G + G, s * nq:(s + 1) * nq].double().reshape(G * nq, -1)
            last = (n - nq + torch.arange(nq, device="cuda")).repeat(G)
            seen = torch.arange(n, device="cuda")[None, :] <= last[:, None]
            z = ((x @ keys[h, r0:r0 + n].T) * st["scale"]).masked_fill(~seen, -math.inf)
            e = torch.logsumexp(z, dim=1)
            w = torch.exp(z - torch.where(e == -math.inf, 0.0, e)[:, None])
            out[h * G:h * G + G, s * nq:(s + 1) * nq] = (w @ values[h, r0:r0 + n]).reshape(G, nq, -1)
            lse[h * G:h * G + G, s * nq:(s + 1) * nq] = e.reshape(G, nq)
            if st["mass"] is not None:
                mass[h, r0:r0 + n] = w.sum(dim=0) + st["mass"][h, r0:r0 + n].double()
    got = {"out": out, "lse": lse}
    return dict(got, mass=mass) if st["mass"] is not None else got


def _exact_mass(st):
    """One query head at a time, over all of its keys, in slabs of queries."""
    c = st["case"]
    W, sink, G = c["window"], c["sink"], c["group"]
    mass = torch.zeros((c["heads"], int(st["cu_k"][-1])), dtype=torch.float64, device="cuda")
    for s, (n, m) in enumerate(zip(st["lens"], st["nq"])):
        k0, q0 = int(st["cu_k"][s]), int(st["cu_q"][s])
        for hq in range(c["heads"] * G):
            k = st["k"][hq // G, k0:k0 + n].double()
            for a in range(0, m, 4096):
                b, end = min(m, a + 4096), n - m + min(m, a + 4096)
                p, j = torch.arange(n - m + a, end, device="cuda")[:, None], torch.arange(end, device="cuda")
                z = st["q"][hq, q0 + a:q0 + b].double() @ k[:end].T * st["scale"]
                hidden = (j > p) | ((j <= p - W) & (j >= sink))
                w = torch.exp(z - st["lse"][hq, q0 + a:q0 + b].double()[:, None]).masked_fill(hidden, 0.0)
                mass[hq // G, k0:k0 + end] += w.sum(dim=0)
    return {"mass": mass}


def exact(case, seed):
    """The outputs in 64 bits.  None where the loops would take too long."""
    kind, lens, d = case["kind"], _lens(case), case["d"]
    H, G = case["heads"], case["group"]
    if kind == "mass":
        pairs = sum(n * m for n, m in zip(lens, _queries(case, lens)))
        if H * G * pairs > 4e10 or H * G * len(lens) > 4200:
            return None
        return _exact_mass(prepare(case, seed))
    if H * sum(lens) * d > 1.5e9 or H * len(lens) > 4200:
        return None
    st = prepare(case, seed)
    if kind == "compact8":
        C = int(st["cu_rows"][-1])
        out = {"len": None, "pos": None}
        for name in ("keys", "values"):
            out[name] = torch.zeros((H, C, d), dtype=torch.float64, device="cuda")
        if st["mass"] is not None:
            out["mass"] = torch.zeros((H, C), dtype=torch.float64, device="cuda")
        for h in range(H):
            for s, n in enumerate(lens):
                a, r = int(st["cu"][s]), int(st["cu_rows"][s])
                kept = a + st["retained"][h, a:a + n].nonzero().squeeze(1)
                for name in ("keys", "values"):
                    out[name][h, r:r + len(kept)] = _exact_8bit(st[name][h, kept].double())
                if st["mass"] is not None:
                    out["mass"][h, r:r + len(kept)] = st["mass"][h, kept].double()
        return out
    keys, values = _exact_rows(st["cache"])
    if kind == "attn8":
        return _exact_attn8(st, keys, values, st["len"].tolist(), case["nq"])
    if kind == "step8":
        out = {n: torch.zeros((H, BLOCK * len(lens), d), dtype=torch.float64, device="cuda") for n in ("keys", "values")}
        count = st["len"].tolist()
        for h in range(H):
            for s in range(len(lens)):
                n, r0 = count[h][s], int(st["cu_rows"][s])
                a = n // BLOCK * BLOCK
                for name, x, b in (("keys", keys, st["cache"]["k_scales"]), ("values", values, st["cache"]["v_scales"])):
                    new = st[name][h, s].double()
                    frac, power = torch.frexp(new.abs().max())
                    e = max(-126, int(power) - 7 + (float(frac) >= 127.5 / 128)) if float(frac) > 0 else -126
                    if n > a:
                        e = max(e, int(b[h, (r0 + a) // BLOCK]) - 127)
                    x[h, r0 + a:r0 + n] = torch.round(x[h, r0 + a:r0 + n] * 2.0 ** -e) * 2.0 ** e
                    x[h, r0 + n] = torch.round(new * 2.0 ** -e) * 2.0 ** e
                    out[name][h, s * BLOCK:s * BLOCK + n + 1 - a] = x[h, r0 + a:r0 + n + 1]
                count[h][s] = n + 1
        return dict(_exact_attn8(st, keys, values, count, 1), len=None, **out)
    C2 = int(st["cu_to"][-1])
    out = {"len": None, "pos": None, "mass": torch.zeros((H, C2), dtype=torch.float64, device="cuda")}
    for name in ("keys", "values"):
        out[name] = torch.zeros((H, C2, d), dtype=torch.float64, device="cuda")
    for h in range(H):
        for s in range(len(lens)):
            rows, r0, to = _kept_rows(st, h, s), int(st["cu_rows"][s]), int(st["cu_to"][s])
            out["mass"][h, to:to + len(rows)] = st["mass"][h, r0 + rows].double()
            for name, x in (("keys", keys), ("values", values)):
                out[name][h, to:to + len(rows)] = _exact_8bit(x[h, r0 + rows])
    return out
