"""The operators of a model's layer around the cache that this library evicts from, as cases that can
be timed and compared: the norm and rotation that make the cached keys, attention over the window
and the sinks of a cache, the compaction into a 4-bit cache, and decoding over that cache.

Kinds:
  rope      per-head RMS norm of queries and keys and the rotary embedding, in one pass
  attn      causal attention that sees a sliding window and the first tokens (sinks)
  compact4  the retained keys and values gathered into a 4-bit cache, and read back
  attn4     attention of a few query tokens over a 4-bit cache
  step      one layer's decode step: norm and rotation, append to the 4-bit cache, attention

Shapes are those of the repository's workloads (8 KV heads a layer, 36x8 heads for whole models,
d 128 and 64, 512 to 128k tokens, 64 ragged prompts), with 4 query heads to a KV head.

A 4-bit cache holds, per (head, row) and 32 channels, a scale 2^(byte - 127) and 32 codes of one
sign, two exponent and one mantissa bit (0, .5, 1, 1.5, 2, 3, 4, 6):
  k_codes  (H, C, d/2)       byte b of a row: channel 2b in the low nibble, 2b + 1 in the high one
  k_scales (H, C, d/32)
  v_codes  (H, C/8, d, 4)    blocks of 8 rows: byte b of a channel holds rows 2b (low) and 2b + 1;
                             slot 64 a + 4 i + n holds channel 64 a + 16 n + i
  v_scales (H, C/8, d/32, 8)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 1.0e6


def _case(name, kind, **kw):
    c = {"kind": kind, "heads": 8, "group": 4, "seqs": 1, "lo": 1, "hi": 1, "d": 128, "dtype": "bf16",
         "nq": 1, "window": 0, "sink": 4, "frac": 0.5, "norm": True, "token_major": True, "len_seed": 0}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of each of 64 sequences, a decode step's queries and keys
        _case("rope_decode_64", "rope", lo=64, hi=64),
        # a 32k prompt's queries and keys as the projections leave them (token major)
        _case("rope_prefill_32k", "rope", lo=32768, hi=32768),
        # fp32, d 64, no norm (a model that only rotates), an odd length
        _case("rope_f32_d64", "rope", lo=4001, hi=4001, d=64, dtype="f32", norm=False),
        # the streaming policy's decode step: 64 ragged sequences, one query each
        _case("attn_decode_64x", "attn", seqs=64, lo=1024, hi=4096, nq=1, window=1024),
        # a prompt of 8k tokens, d 64, full causal attention
        _case("attn_prefill_8k_d64", "attn", lo=8192, hi=8192, nq=0, d=64, window=8192, sink=0),
        # a prompt of 32k tokens under the streaming policy, and the largest work listed
        _case("attn_prefill_32k", "attn", lo=32768, hi=32768, nq=0, window=4096),
        # fp32, ragged prompts in one batch
        _case("attn_f32_ragged", "attn", heads=8, group=1, seqs=5, lo=150, hi=1500, nq=0, d=64, dtype="f32",
              window=128),
        # one layer's repaired cache of an odd length into 4 bits
        _case("compact4_layer_4k", "compact4", lo=4001, hi=4001),
        # a whole 36-layer model's cache into 4 bits
        _case("compact4_36x8x16k", "compact4", heads=288, lo=16384, hi=16384, frac=0.4),
        # the smallest decode step: one sequence, one layer, a cache of 512 rows
        _case("step_512", "step", lo=512, hi=512),
        # a decode step of 64 ragged sequences
        _case("step_64x", "step", seqs=64, lo=1024, hi=4096),
        # one layer at 128k cached rows, a few speculative tokens
        _case("attn4_layer_128k", "attn4", lo=131072, hi=131072, nq=4),
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
    """A case of the same ranges: 1 to 32k tokens to rotate, prompts and caches from a few tokens to
    128k, one sequence or a ragged batch, both head sizes and types, 1 to 8 query heads a KV head."""
    top = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rope", "attn", "attn", "compact4", "attn4", "step"])
        seqs = rng.choice([1, 1, 2, 5, 16, 64])
        longest = {"rope": 32768, "attn": 32768, "compact4": 32768, "attn4": 131072, "step": 131072}[kind]
        if kind == "rope":
            seqs = 1
        hi = _log(rng, 1 if kind == "rope" else 16, longest)
        lo = hi if seqs == 1 else max(1, int(hi * rng.choice([0.05, 0.25, 0.7])))
        heads = rng.choice([1, 8, 8, 40, 288]) if kind == "compact4" else rng.choice([2, 8, 8, 8])
        nq = {"attn": rng.choice([0, 0, 1, _log(rng, 2, 512)]), "attn4": rng.choice([1, 1, 2, 7])}.get(kind, 1)
        c = _case(None, kind, heads=heads, group=rng.choice([1, 2, 4, 4, 8]), seqs=seqs, lo=lo, hi=hi,
                  d=rng.choice([64, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), nq=nq,
                  window=_log(rng, 16, hi) if kind == "attn" and hi > 16 else hi, sink=rng.choice([0, 4, 16]),
                  frac=rng.choice([0.1, 0.3, 0.5, 0.7]), norm=rng.choice([True, True, False]),
                  token_major=rng.choice([True, True, False]), len_seed=rng.randrange(1 << 20))
        elements = heads * c["group"] * sum(_lens(c)) * c["d"]
        if _cost(c) * (8 if c["dtype"] == "f32" else 1) <= 0.5 * top and elements <= 1.2e9:
            return c


# ---------------------------------------------------------------- the 4-bit format, plainly

def _quantise(x):
    """Codes (uint8, x's shape) and scale bytes (uint8, one per 32 channels) of (..., d) fp32 values."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = g.abs().amax(dim=-1, keepdim=True)
    ok = torch.isfinite(amax)
    g, amax = torch.where(ok, g, 0.0), torch.where(ok, amax, 0.0)
    byte = (((amax.view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 252)
    a = g.abs() * ((254 - byte) << 23).view(torch.float32)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = torch.where(g < 0, code + 8, code)
    return code.reshape(x.shape), byte.squeeze(-1).to(torch.uint8)


def _values(code, byte):
    """What codes (..., d) under scale bytes (..., d/32) stand for, in fp32."""
    mag = (code & 7).to(torch.int32)
    e, m = mag >> 1, (mag & 1).to(torch.float32)
    v = torch.where(e > 0, (1.0 + 0.5 * m) * torch.exp2((e - 1).to(torch.float32)), 0.5 * m)
    v = torch.where(code >= 8, -v, v)
    scale = (byte.to(torch.int32) << 23).view(torch.float32)
    return (v.reshape(*byte.shape, 32) * scale.unsqueeze(-1)).reshape(code.shape)


def _pack(kc, kb, vc, vb):
    """The cache's arrays from codes (H, C, d) and scale bytes (H, C, d/32) of keys and values."""
    H, C, d = kc.shape
    k_codes = kc[..., 0::2] | (kc[..., 1::2] << 4)
    v = vc.reshape(H, C // 8, 4, 2, d)
    v = (v[:, :, :, 0] | (v[:, :, :, 1] << 4)).reshape(H, C // 8, 4, d // 64, 4, 16)
    v_codes = v.permute(0, 1, 3, 5, 4, 2).reshape(H, C // 8, d, 4).contiguous()
    v_scales = vb.reshape(H, C // 8, 8, d // 32).transpose(2, 3).contiguous()
    return {"k_codes": k_codes.contiguous(), "k_scales": kb.contiguous(), "v_codes": v_codes, "v_scales": v_scales}


def _unpack(c):
    """Keys and values (H, C, d) in fp32 of a cache's arrays."""
    H, C, half = c["k_codes"].shape
    d = 2 * half
    kc = torch.stack([c["k_codes"] & 15, c["k_codes"] >> 4], dim=-1).reshape(H, C, d)
    v = c["v_codes"].reshape(H, C // 8, d // 64, 16, 4, 4).permute(0, 1, 5, 2, 4, 3).reshape(H, C // 8, 4, d)
    vc = torch.stack([v & 15, v >> 4], dim=3).reshape(H, C, d)
    vb = c["v_scales"].transpose(2, 3).reshape(H, C, d // 32)
    return _values(kc, c["k_scales"]), _values(vc, vb)


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


def _rope_table(n, d):
    f = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _cum(x):
    return np.concatenate([[0], np.cumsum(x)]).astype(np.int64)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))
    lens, H, G, d, kind, dt = _lens(case), case["heads"], case["group"], case["d"], case["kind"], _dtype(case)
    st = {"case": case, "lens": lens, "scale": d ** -0.5}
    if kind in ("rope", "step"):
        T = sum(lens) if kind == "rope" else len(lens)
        st["q"], st["k"] = _heads_of(case, g, H * G, T), _heads_of(case, g, H, T)
        st["qw"] = 1.0 + 0.1 * _randn(g, d) if case["norm"] else None
        st["kw"] = 1.0 + 0.1 * _randn(g, d) if case["norm"] else None
        st["table"] = _rope_table(max(lens) + 1, d)
        # a decode step's tokens stand at the ends of their sequences, a prompt's one after another
        st["pos"] = torch.tensor(lens, dtype=torch.int32, device="cuda") if kind == "step" else \
            torch.arange(T, dtype=torch.int32, device="cuda")
    if kind == "attn":
        nq, T = _queries(case, lens), sum(lens)
        st["nq"], st["cu_q"], st["cu_k"] = nq, _cum(nq), _cum(lens)
        st["q"], st["k"] = _randn(g, H * G, sum(nq), d).to(dt), _keys(case, g, H, T)
        st["v"] = _randn(g, H, T, d).to(dt)
    if kind == "compact4":
        T, st["cu"] = sum(lens), _cum(lens)
        budget = [int(case["frac"] * n) for n in lens]
        st["keys"], st["values"] = _keys(case, g, H, T), _randn(g, H, T, d).to(dt)
        score, st["retained"] = torch.rand((H, T), generator=g, device="cuda"), torch.zeros((H, T), dtype=torch.uint8, device="cuda")
        for a, n, b in zip(st["cu"], lens, budget):
            st["retained"][:, a:a + n].scatter_(1, score[:, a:a + n].topk(b, dim=1).indices, 1)
        st["cu_rows"] = _cum([(b + 31) // 32 * 32 for b in budget])
        C = int(st["cu_rows"][-1])
        # the cache that a program reserves once
        st["cache"] = {"k_codes": torch.zeros((H, C, d // 2), dtype=torch.uint8, device="cuda"),
                       "k_scales": torch.zeros((H, C, d // 32), dtype=torch.uint8, device="cuda"),
                       "v_codes": torch.zeros((H, C // 8, d, 4), dtype=torch.uint8, device="cuda"),
                       "v_scales": torch.zeros((H, C // 8, d // 32, 8), dtype=torch.uint8, device="cuda")}
    if kind in ("attn4", "step"):
        st["cu_rows"] = _cum([(n + case["nq"] + 31) // 32 * 32 for n in lens])
        C = int(st["cu_rows"][-1])
        packed = [_quantise(x) for x in (_keys(case, g, H, C).float(), _randn(g, H, C, d).to(dt).float())]
        st["cache"] = _pack(*packed[0], *packed[1])
        # heads of one layer keep the same number of rows, or a few less
        less = torch.randint(0, 9, (H, len(lens)), generator=g, device="cuda", dtype=torch.int32)
        st["len"] = (torch.tensor(lens, dtype=torch.int32, device="cuda") - less).clamp(min=1)
    if kind == "attn4":
        st["cu_q"] = np.arange(len(lens) + 1, dtype=np.int64) * case["nq"]
        st["q"] = _randn(g, H * G, len(lens) * case["nq"], d).to(dt)
    if kind == "step":
        st["cu_q"] = np.arange(len(lens) + 1, dtype=np.int64)
        st["values"] = _heads_of(case, g, H, len(lens))
    return st


# ---------------------------------------------------------------- the plain forms

def _softmax_product(q, k, v, mask, scale):
    """softmax of scale q k^T over the places that mask leaves, times v, in fp32; 0 and -inf for rows
    that it leaves nothing."""
    s = torch.where(mask, torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale, -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - m)
    l = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(l > 0, l, 1.0), (torch.log(l) + m).squeeze(-1)


def _norm_rope(x, w, table, pos):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w
    cs = table[pos.long()]
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cs[:, :h], cs[:, h:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _plain_attn(st):
    c, lens, nq = st["case"], st["lens"], st["nq"]
    H, G, S, W, sink, d = c["heads"], c["group"], len(lens), c["window"], c["sink"], c["d"]
    dev, longest, top = "cuda", max(nq), max(lens)
    n, m = torch.tensor(lens, device=dev)[:, None], torch.tensor(nq, device=dev)[:, None]
    k0, q0 = torch.tensor(st["cu_k"][:-1], device=dev)[:, None], torch.tensor(st["cu_q"][:-1], device=dev)[:, None]
    out = torch.empty((H * G, int(st["cu_q"][-1]), d), dtype=_dtype(c), device=dev)
    lse = torch.empty((H * G, int(st["cu_q"][-1])), dtype=torch.float32, device=dev)
    step = 1 << max(0, int(math.log2(max(1, 2 ** 27 // (S * H * G * min(top, W + 1024))))))
    # blocks of queries, counted from the sequences' ends so that their windows lie alike: the scores
    # of all blocks at once would not fit
    for a in range(0, longest, min(step, 1024)):
        b = min(longest, a + min(step, 1024))
        i = torch.arange(a, b, device=dev)[None, :] + (m - longest)          # (S, rows) query tokens
        p = n - m + i
        cols = min(max(W - 1, 0) + b - a, top - longest + b)
        j = (n - longest + b - cols) + torch.arange(cols, device=dev)[None, :]
        js = torch.arange(sink, device=dev)[None, :].expand(S, sink)
        far = p[:, :, None] - j[:, None, :]
        near = (far >= 0) & (far < W) & (j >= sink)[:, None, :]
        first = (js[:, None, :] <= p[:, :, None])
        mask = torch.cat([first, near], dim=2)                                # (S, rows, cols)
        at = (k0 + torch.cat([torch.minimum(js, n - 1), j.clamp(min=0)], dim=1)).reshape(-1)
        kk = st["k"][:, at].float().reshape(H, S, -1, d)
        vv = st["v"][:, at].float().reshape(H, S, -1, d)
        qq = st["q"][:, (q0 + i.clamp(min=0)).reshape(-1)].float().reshape(H, G, S, b - a, d).transpose(1, 2)
        o, e = _softmax_product(qq.reshape(H, S, G * (b - a), d), kk, vv,
                                mask[:, None].expand(S, G, b - a, -1).reshape(S, G * (b - a), -1), st["scale"])
        o = o.reshape(H, S, G, b - a, d).transpose(1, 2).reshape(H * G, S * (b - a), d)
        e = e.reshape(H, S, G, b - a).transpose(1, 2).reshape(H * G, S * (b - a))
        live = (i >= 0).reshape(-1)
        to = (q0 + i).reshape(-1)[live]
        out[:, to] = o[:, live].to(out.dtype)
        lse[:, to] = e[:, live]
    return {"out": out, "lse": lse}


def _plain_compact4(st):
    c, lens = st["case"], st["lens"]
    H, dev = c["heads"], "cuda"
    C, T = int(st["cu_rows"][-1]), int(st["cu"][-1])
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
        x = torch.zeros((H, C, c["d"]), dtype=_dtype(c), device=dev)
        x[h, row] = _values(*_quantise(st[name][h, t].float())).to(x.dtype)
        out[name] = x
    return out


def _plain_attn4(q, keys, values, length, cu_rows, nq, scale, dtype):
    """q (H*G, S*nq, d) over keys and values (H, C, d) in fp32; length (H, S) counts the rows."""
    H, C, d = keys.shape
    S, dev = len(cu_rows) - 1, "cuda"
    G, top = q.shape[0] // H, int((cu_rows[1:] - cu_rows[:-1]).max())
    j = torch.arange(top, device=dev)
    at = (torch.tensor(cu_rows[:-1], device=dev)[:, None] + j).clamp(max=C - 1).reshape(-1)
    i = torch.arange(nq, device=dev)
    mask = j < (length[:, :, None, None] - (nq - 1 - i)[:, None])             # (H, S, nq, top)
    qq = q.float().reshape(H, G, S, nq, d).transpose(1, 2).reshape(H, S, G * nq, d)
    o, e = _softmax_product(qq, keys[:, at].reshape(H, S, top, d), values[:, at].reshape(H, S, top, d),
                            mask[:, :, None].expand(H, S, G, nq, top).reshape(H, S, G * nq, top), scale)
    o = o.reshape(H, S, G, nq, d).transpose(1, 2).reshape(H * G, S * nq, d)
    return o.to(dtype), e.reshape(H, S, G, nq).transpose(1, 2).reshape(H * G, S * nq)


def _plain(st):
    c = st["case"]
    kind, dt = c["kind"], _dtype(c)
    if kind == "rope":
        return {"q": _norm_rope(st["q"], st["qw"], st["table"], st["pos"]).to(dt),
                "k": _norm_rope(st["k"], st["kw"], st["table"], st["pos"]).to(dt)}
    if kind == "attn":
        return _plain_attn(st)
    if kind == "compact4":
        return _plain_compact4(st)
    keys, values = _unpack(st["cache"])
    if kind == "attn4":
        o, e = _plain_attn4(st["q"], keys, values, st["len"], st["cu_rows"], c["nq"], st["scale"], dt)
        return {"out": o, "lse": e}
    q = _norm_rope(st["q"], st["qw"], st["table"], st["pos"]).to(dt)
    k = _norm_rope(st["k"], st["kw"], st["table"], st["pos"]).to(dt)
    new_k, new_v = _values(*_quantise(k.float())), _values(*_quantise(st["values"].float()))
    row = torch.tensor(st["cu_rows"][:-1], device="cuda") + st["len"]
    h = torch.arange(c["heads"], device="cuda")[:, None]
    keys[h, row], values[h, row] = new_k, new_v
    length = st["len"] + 1
    o, e = _plain_attn4(q, keys, values, length, st["cu_rows"], 1, st["scale"], dt)
    return {"out": o, "lse": e, "len": length, "new_keys": new_k.to(dt), "new_values": new_v.to(dt)}


# ---------------------------------------------------------------- the framework's calls

def _framework(st):
    from paper_2608_27128_amd import binding

    c = st["case"]
    kind, dt = c["kind"], _dtype(c)
    if kind == "rope":
        return binding.qk_norm_rope(st["q"], st["k"], st["qw"], st["kw"], EPS, st["table"], st["pos"])
    if kind == "attn":
        return binding.sink_attention(st["q"], st["k"], st["v"], c["window"], c["sink"], st["scale"],
                                      st["cu_q"], st["cu_k"], want_lse=True)
    cache = binding.Cache4(cu_rows=st["cu_rows"], **st["cache"])
    if kind == "compact4":
        got = binding.cache4_compact(st["keys"], st["values"], st["retained"], cache, st["cu"])
        kv = binding.cache4_read(cache, got["len"], dt)
        return {"len": got["len"], "pos": got["pos"], "keys": kv["keys"], "values": kv["values"]}
    if kind == "attn4":
        return binding.cache4_attention(st["q"], cache, st["len"], st["scale"], st["cu_q"], want_lse=True)
    r = binding.qk_norm_rope(st["q"], st["k"], st["qw"], st["kw"], EPS, st["table"], st["pos"])
    grown = binding.cache4_append(r["k"], st["values"], cache, st["len"], st["cu_q"])
    got = binding.cache4_attention(r["q"], cache, grown["len"], st["scale"], st["cu_q"], want_lse=True)
    new = binding.cache4_read(cache, grown["len"], dt, first=st["len"], cu_out=st["cu_q"])
    return {"out": got["out"], "lse": got["lse"], "len": grown["len"], "new_keys": new["keys"],
            "new_values": new["values"]}


def run(st):
    return _framework(st) if own else _plain(st)


# ---------------------------------------------------------------- what a pass cannot do without

def _visible(case):
    """Pairs of a query token and a key that it sees, and keys that any query sees, over all sequences."""
    pairs = keys = 0
    for n, m in zip(_lens(case), _queries(case, _lens(case))):
        p = np.arange(n - m, n, dtype=np.float64)
        pairs += float(np.minimum(p + 1, min(case["sink"], n) + np.minimum(case["window"], np.maximum(0, p + 1 - case["sink"]))).sum())
        keys += min(n, case["sink"] + case["window"] + m - 1)
    return pairs, keys


def work(case):
    H, G, d, kind, lens = case["heads"], case["group"], case["d"], case["kind"], _lens(case)
    e = 4.0 if case["dtype"] == "f32" else 2.0
    T, S = float(sum(lens)), float(len(lens))
    if kind == "rope":
        return {"bytes": T * (2.0 * H * (G + 1) * d * e + 4.0 * d + 4.0), "flops": T * H * (G + 1) * d * 9.0}
    if kind == "attn":
        pairs, keys = _visible(case)
        n = float(sum(_queries(case, lens)))
        return {"bytes": H * (2.0 * G * n * d * e + 4.0 * G * n + 2.0 * keys * d * e), "flops": 4.0 * d * pairs * H * G}
    row = 2.0 * (d / 2 + d / 32)                      # a cached key and value, in bytes
    if kind == "compact4":
        kept = float(H * sum(int(case["frac"] * n) for n in lens))
        return {"bytes": kept * (2.0 * d * e + row + 4.0) + kept * (row + 2.0 * d * e) + H * T, "flops": kept * d * 8.0}
    n = case["nq"] * S
    got = {"bytes": H * (T * row + 2.0 * G * n * d * e + 4.0 * G * n), "flops": 4.0 * d * T * H * G * case["nq"]}
    if kind == "step":
        got["bytes"] += S * (2.0 * H * (G + 1) * d * e + 4.0 * d) + H * S * (2.0 * d * e + row)
    return got


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---------------------------------------------------------------- the definition in 64 bits

def _grid():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")


def _exact_4bit(x):
    """The value that (..., d) 64-bit numbers have in 4 bits: the nearest on the grid, ties to the even code."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = g.abs().amax(dim=-1, keepdim=True)
    frac, power = torch.frexp(amax)
    e = torch.clamp(power - 3 + (frac >= 0.875).int(), -126, 125)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).double()
    a = (g.abs() / torch.exp2(e)).clamp(max=6.0)
    grid = _grid()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    code = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (grid[code] * torch.sign(g) * torch.exp2(e)).reshape(x.shape)


def _exact_softmax(q, k, v, seen, scale):
    s = ((q @ k.T) * scale).masked_fill(~seen, -math.inf)
    e = torch.logsumexp(s, dim=1)
    w = torch.exp(s - torch.where(e == -math.inf, torch.zeros_like(e), e)[:, None])
    return w @ v, e


def _exact_rope(x, w, table, pos):
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(dim=-1, keepdim=True) + EPS).sqrt() * w.double()
    z = torch.complex(*x.chunk(2, dim=-1)) * torch.complex(*table.double()[pos.long()].chunk(2, dim=-1))
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_attn4(q, keys, values, length, cu_rows, nq, scale):
    H = keys.shape[0]
    G = q.shape[0] // H
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    count = length.tolist()
    for h in range(H):
        for s in range(len(cu_rows) - 1):
            r0, n = int(cu_rows[s]), count[h][s]
            k, v = keys[h, r0:r0 + n], values[h, r0:r0 + n]
            last = n - nq + torch.arange(nq, device="cuda")
            seen = torch.arange(n, device="cuda")[None, :] <= last[:, None]
            for hq in range(h * G, h * G + G):
                o, e = _exact_softmax(q[hq, s * nq:(s + 1) * nq].double(), k, v, seen, scale)
                out[hq, s * nq:(s + 1) * nq], lse[hq, s * nq:(s + 1) * nq] = o, e
    return out, lse


def exact(case, seed):
    """The outputs in 64 bits: bf16 steps between operators stay, since they are values that a program
    holds.  None where the loops would take too long."""
    kind, lens, d = case["kind"], _lens(case), case["d"]
    H, G = case["heads"], case["group"]
    if H * G * sum(lens) * d > 1.5e9 or (kind != "rope" and H * len(lens) * (G if "attn" in kind or kind == "step" else 1) > 4200):
        return None
    st = prepare(case, seed)
    if kind == "rope":
        return {n: _exact_rope(st[n], st[n + "w"], st["table"], st["pos"]) for n in ("q", "k")}
    if kind == "attn":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(st["q"].shape[:2], dtype=torch.float64, device="cuda")
        W, sink = case["window"], case["sink"]
        for s, (n, m) in enumerate(zip(lens, st["nq"])):
            k0, q0 = int(st["cu_k"][s]), int(st["cu_q"][s])
            for h in range(H):
                k, v = st["k"][h, k0:k0 + n].double(), st["v"][h, k0:k0 + n].double()
                for a in range(0, m, 2048):
                    b = min(m, a + 2048)
                    p = torch.arange(n - m + a, n - m + b, device="cuda")[:, None]
                    lo = max(0, n - m + a - W) if n - m + a - W > sink else 0
                    j = torch.cat([torch.arange(min(sink, lo), device="cuda"), torch.arange(lo, n - m + b, device="cuda")])
                    seen = (j <= p) & ((p - j < W) | (j < sink))
                    for hq in range(h * G, h * G + G):
                        o, e = _exact_softmax(st["q"][hq, q0 + a:q0 + b].double(), k[j], v[j], seen, st["scale"])
                        out[hq, q0 + a:q0 + b], lse[hq, q0 + a:q0 + b] = o, e
        return {"out": out, "lse": lse}
    if kind == "compact4":
        C = int(st["cu_rows"][-1])
        out = {"len": None, "pos": None}
        for name in ("keys", "values"):
            x = torch.zeros((H, C, d), dtype=torch.float64, device="cuda")
            for h in range(H):
                for s, n in enumerate(lens):
                    a, r = int(st["cu"][s]), int(st["cu_rows"][s])
                    kept = st["retained"][h, a:a + n].nonzero().squeeze(1)
                    x[h, r:r + len(kept)] = _exact_4bit(st[name][h, a + kept].double()) if len(kept) else 0.0
            out[name] = x
        return out
    keys, values = (x.double() for x in _unpack(st["cache"]))     # exact: a code times a power of two
    if kind == "attn4":
        o, e = _exact_attn4(st["q"], keys, values, st["len"], st["cu_rows"], case["nq"], st["scale"])
        return {"out": o, "lse": e}
    # the step's own roundings (the rotated query and key, the new rows in 4 bits) can fall either way
    # where 32 and 64 bits lie on two sides of a tie: what follows from them has no one value
    return {"out": None, "lse": None, "len": None, "new_keys": None,
            "new_values": _exact_4bit(st["values"].double())}
