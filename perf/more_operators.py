"""Operators that let a decode step read fewer bytes of its caches: cases, plain forms and exact values.

pack     new rows of K and V written into 4-bit caches, and read back: groups of 32 elements share a step and a
         lowest value in fp16, low + step * code with codes 0..15.
attend4  attention of the newest ``n_q`` queries of every sequence over its 4-bit cache (a length per KV head,
         causal among the new tokens), with each cached key's attention weight added to an accumulator.
window   attention over bf16 caches where a query sees the ``window`` newest rows and the ``n_sink`` first ones.
evict4   4-bit caches are cut to their budget by accumulated weight and compacted into the decode caches.

``run`` is the plain form (elementary torch operations in 32 bits, 64 where a code is chosen) unless ``own`` is
set, and then the framework's operators.

A row of a 4-bit cache of head_dim d holds d / 8 words of 32 bits with eight codes each, the first in the lowest four
bits.  Word t d / 32 + g of a row of K (t < 4) holds elements 32 g + 8 t .. 32 g + 8 t + 7; word w of a row of V holds
elements w, w + d / 8, .., w + 7 d / 8.  A row's scales are fp16 [2 (K, V)][d / 32][2 (step, low)].
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 32
TOP = 65504.0  # largest finite fp16


# ------------------------------------------------------------------------------------------ cases
def _pack(name, b, hkv, d, cap, n, lo, hi):
    return {"name": name, "op": "pack", "b": b, "hkv": hkv, "d": d, "cap": cap, "n": n, "lo": lo, "hi": hi}


def _attend4(name, b, hq, hkv, d, cap, n_q, lo, hi, weights):
    return {"name": name, "op": "attend4", "b": b, "hq": hq, "hkv": hkv, "d": d, "cap": cap, "n_q": n_q, "lo": lo,
            "hi": hi, "weights": weights}


def _window(name, b, hq, hkv, d, cap, n_q, lo, hi, window, n_sink):
    return {"name": name, "op": "window", "b": b, "hq": hq, "hkv": hkv, "d": d, "cap": cap, "n_q": n_q, "lo": lo,
            "hi": hi, "window": window, "n_sink": n_sink}


def _evict4(name, layers, b, hkv, d, cap, cap_out, lo, hi, budget, n_prefix, window):
    return {"name": name, "op": "evict4", "layers": layers, "b": b, "hkv": hkv, "d": d, "cap": cap,
            "cap_out": cap_out, "lo": lo, "hi": hi, "budget": budget, "n_prefix": n_prefix, "window": window}


def listed():
    return [
        # one decode step's new row in every cache of a layer, Qwen3-4B shape: latency only
        _pack("pack_token", 16, 8, 128, 4224, 1, 4097, 4224),
        # prompts of many lengths moved from their bf16 caches into 4-bit ones
        _pack("pack_prompt", 8, 8, 128, 8320, 8203, 1031, 8203),
        # one token of one short sequence, the smallest shape of the workloads: latency only
        _attend4("attend4_tiny", 1, 4, 2, 64, 1088, 1, 1088, 1088, True),
        # one layer of a decode step between two evictions, Qwen3-4B shape
        _attend4("attend4_step", 16, 32, 8, 128, 4224, 1, 4097, 4224, True),
        # one token of a few long sequences of very different lengths, five query heads per group
        _attend4("attend4_long", 4, 40, 8, 128, 32768, 1, 1, 32768, False),
        # a few draft tokens per sequence, head_dim 64, odd lengths, caches shorter than the draft
        _attend4("attend4_draft", 7, 32, 8, 64, 8320, 7, 5, 8317, True),
        # one piece of a long prompt that is taken in pieces, over what was packed before it
        _attend4("attend4_piece", 1, 32, 8, 128, 32768, 512, 32000, 32768, False),
        # one token of short sequences with a narrow window, some not yet as long as it
        _window("window_tiny", 2, 4, 2, 64, 1088, 1, 0, 1088, 128, 4),
        # one layer of a decode step of long sequences whose caches are not cut, window and first tokens
        _window("window_step", 16, 32, 8, 128, 8320, 1, 1031, 8203, 1024, 4),
        # a whole prompt through a layer with a window
        _window("window_prompt", 1, 32, 8, 128, 8320, 8192, 8192, 8192, 1024, 4),
        # long prompts of many lengths cut into smaller decode caches, some of them already under the budget
        _evict4("evict4_prompt", 5, 8, 8, 128, 32768, 2176, 1, 32768, 2048, 4, 32),
        # eight layers of the Qwen3-4B shape, one period's worth of rows evicted from every cache
        _evict4("evict4_period", 8, 16, 8, 128, 4224, 4224, 4224, 4224, 4096, 0, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    d = rng.choice((64, 128))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 4, 5, 7, 8))
    kind = rng.choice(("pack", "token4", "draft4", "piece4", "token", "draft", "prompt", "evict4"))
    if kind == "pack":
        b = _log(rng, 1, 16)
        cap = _log(rng, 16, min(32768, 8 * 8320 * 8 // (b * hkv)))
        n = rng.choice((1, 1, rng.randint(1, cap), cap))
        lo = rng.randint(0, cap)
        c = _pack("", b, hkv, d, cap, n, lo, rng.randint(max(lo, 1), cap))
    elif kind in ("token4", "draft4"):
        b = _log(rng, 1, 16)
        cap = _log(rng, 64, min(32768, 16 * 4224 * 8 // (b * hkv)))
        lo = rng.randint(0, cap)
        n_q = 1 if kind == "token4" else rng.randint(2, 24)
        c = _attend4("", b, hq, hkv, d, cap, n_q, lo, rng.randint(max(lo, 1), cap), rng.random() < 0.5)
    elif kind == "piece4":
        n_q = _log(rng, 25, 512)
        b = _log(rng, 1, 4)
        cap = rng.randint(n_q, max(n_q, min(32768, 32 * 512 * 32768 // (b * hq * n_q))))
        lo = rng.randint(cap // 2, cap)
        c = _attend4("", b, hq, hkv, d, cap, n_q, lo, rng.randint(lo, cap), rng.random() < 0.5)
    elif kind in ("token", "draft"):
        b = _log(rng, 1, 32)
        cap = _log(rng, 64, min(32768, 16 * 8320 * 8 // (b * hkv)))
        lo = rng.randint(0, cap)
        n_q = 1 if kind == "token" else rng.randint(2, 40)
        c = _window("", b, hq, hkv, d, cap, n_q, lo, rng.randint(max(lo, 1), cap), _log(rng, 1, cap),
                    rng.choice((0, 1, 4, 133)))
    elif kind == "prompt":
        b = _log(rng, 1, 8)
        n_q = _log(rng, 65, min(8192, int(8192 * math.sqrt(16 / (b * hq)))))
        cap = rng.randint(n_q, min(8320, n_q + 1100))
        window = _log(rng, 16, 1024)
        lo = rng.randint(n_q // 2, cap)
        c = _window("", b, hq, hkv, d, cap, n_q, lo, rng.randint(lo, cap), window, rng.choice((0, 1, 4, 133)))
    else:
        layers, b = rng.randint(1, 8), _log(rng, 1, 16)
        cap = _log(rng, 64, min(32768, 8 * 16 * 8 * 4224 // (layers * b * hkv)))
        window = rng.randint(0, min(32, cap // 4))
        n_prefix = rng.choice((0, 1, 4, 7))
        budget = rng.randint(n_prefix + window + 1, cap)
        lo = rng.randint(0, cap)
        c = _evict4("", layers, b, hkv, d, cap, rng.randint(budget, cap), lo, rng.randint(lo, cap), budget, n_prefix,
                    window)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ the 4-bit format
def _to_fp16(x):
    """Nearest fp16 numbers, ties to even, largest magnitude 65504; fp64 by a table, as a conversion by way of fp32
    would round twice."""
    if x.dtype != torch.float64:
        return x.clamp(-TOP, TOP).to(torch.float16).to(x.dtype)
    table = torch.arange(0x7C00, dtype=torch.int16, device=x.device).view(torch.float16).double()
    a = x.abs().clamp(max=TOP)
    hi = torch.searchsorted(table, a)  # the first entry that is not below
    lo = (hi - 1).clamp(min=0)
    below, above = a - table[lo], table[hi] - a
    return torch.copysign(table[torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)], x)


def _quantise(x, dtype):
    """(codes, step, low) of [.., d] values, computed in `dtype`."""
    g = x.to(dtype).unflatten(-1, (-1, GROUP))
    low = _to_fp16(g.amin(-1))
    step = _to_fp16(((g.amax(-1) - low) / 15).clamp(min=0))
    code = torch.round((g - low[..., None]) / torch.where(step > 0, step, torch.inf)[..., None]).clamp(0, 15)
    return code.flatten(-2), step, low


def _words(code, which):
    """Codes [.., d] of rows of K (which: 0) or V (1) as the bytes of their words, [.., d / 2]."""
    n = code.to(torch.uint8)
    if which == 0:
        n = n.unflatten(-1, (-1, 4, 8)).transpose(-2, -3).flatten(-3, -2)
    else:
        n = n.unflatten(-1, (8, -1)).transpose(-1, -2)
    return (n[..., 0::2] | (n[..., 1::2] << 4)).flatten(-2).contiguous()


def _values(packed, scales, which, dtype):
    """Rows of a 4-bit cache as numbers."""
    p = packed.unflatten(-1, (-1, 4))
    code = torch.stack((p & 15, p >> 4), -1).flatten(-2)
    if which == 0:
        code = code.unflatten(-2, (4, -1)).transpose(-2, -3).flatten(-3)
    else:
        code = code.transpose(-1, -2).flatten(-2)
    sc = scales[..., which, :, :].to(dtype)
    g = code.to(dtype).unflatten(-1, (-1, GROUP))
    return (sc[..., 1, None] + sc[..., 0, None] * g).flatten(-2)


def _cache4(gen, d, *lead):
    """A 4-bit cache of random keys (with a mean of their own per head) and values, made in pieces."""
    K4, V4 = (torch.empty(*lead, d // 2, dtype=torch.uint8, device=DEV) for _ in "KV")
    S4 = torch.empty(*lead, 2, d // GROUP, 2, dtype=torch.float16, device=DEV)
    for i in range(lead[0]):
        for which, out in ((0, K4), (1, V4)):
            x = _randn(gen, *lead[1:], d)
            if which == 0:
                x += 0.5 * _randn(gen, lead[-2], 1, d)
            code, step, low = _quantise(x, torch.float32)
            out[i] = _words(code, which)
            S4[i, ..., which, :, 0], S4[i, ..., which, :, 1] = step, low
    return K4, V4, S4


# ------------------------------------------------------------------------------------------ inputs
def _lengths(n, lo, hi):
    """n lengths spread evenly over lo..hi, both ends among them, in a fixed scattered order: the work of a case
    does not depend on the seed."""
    step = next(s for s in range(max(1, int(n * 0.618)), 2 * n + 2) if math.gcd(s, n) == 1)
    return [hi if n == 1 else lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _randn(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    c, st = case, {"case": case}
    b, hkv, d, cap = c["b"], c["hkv"], c["d"], c["cap"]
    lens = _lengths(c.get("layers", 1) * b * hkv, c["lo"], c["hi"])
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["length"] = length.view(b, hkv) if c["op"] != "evict4" else length.view(c["layers"], b, hkv)
    if c["op"] == "pack":
        n = c["n"]
        st["K"], st["V"] = _randn(gen, b, hkv, n, d), _randn(gen, b, hkv, n, d)
        # keys with a mean of their own per head and some channels that stand out, as models' keys have
        st["K"] += 0.5 * _randn(gen, 1, hkv, 1, d)
        st["K"][..., ::37] *= 6
        st["first"] = (st["length"] - n).clamp(min=0).to(torch.int32)
        st["K4"], st["V4"] = (torch.zeros(b, hkv, cap, d // 2, dtype=torch.uint8, device=DEV) for _ in "KV")
        st["S4"] = torch.zeros(b, hkv, cap, 2, d // GROUP, 2, dtype=torch.float16, device=DEV)
        st["K_out"], st["V_out"] = (torch.zeros(b, hkv, n, d, dtype=torch.bfloat16, device=DEV) for _ in "KV")
    elif c["op"] == "attend4":
        st["K4"], st["V4"], st["S4"] = _cache4(gen, d, b, hkv, cap)
        st["weights"] = torch.rand(b, hkv, cap, generator=gen, device=DEV) if c["weights"] else None
    elif c["op"] == "window":
        st["K"], st["V"] = _randn(gen, b, hkv, cap, d), _randn(gen, b, hkv, cap, d)
        st["K"] += 0.5 * _randn(gen, 1, hkv, 1, d)
    else:
        layers, out = c["layers"], c["cap_out"]
        st["K4"], st["V4"] = (torch.randint(0, 256, (layers, b, hkv, cap, d // 2), generator=gen, dtype=torch.uint8,
                                            device=DEV) for _ in "KV")
        st["S4"] = torch.rand(layers, b, hkv, cap, 2, d // GROUP, 2, generator=gen, device=DEV,
                              dtype=torch.float16) - 0.5
        # accumulated weights: heavy-tailed, with many equal small values (rows seen by few queries)
        w = torch.exp(1.5 * _randn(gen, layers, b, hkv, cap, dtype=torch.float32) - 3)
        st["weights"] = torch.where(w < 0.03, torch.round(w * 256) / 256, w)
        st["K4_out"], st["V4_out"], st["S4_out"] = (
            torch.zeros(layers, b, hkv, out, *t.shape[4:], dtype=t.dtype, device=DEV)
            for t in (st["K4"], st["V4"], st["S4"]))
        st["weights_out"] = torch.zeros(layers, b, hkv, out, device=DEV)
    if "n_q" in c:
        st["q"] = _randn(gen, b, c["hq"], c["n_q"], d) * 2
    if own:
        from paper_2609_04971_gb300 import bkv
        keep = c["window"] if c["op"] == "evict4" else 1
        st["bk"] = bkv.BeaconKV(n_layers=c.get("layers", 1), batch=b, n_q_heads=c.get("hq", hkv), n_kv_heads=hkv,
                                head_dim=d, n_beacons=0 if keep else 1, window=keep, capacity=cap,
                                n_prefix=c.get("n_prefix", 0))
        if c["op"] == "attend4":
            st["bk"].reserve_attend4(n_q=c["n_q"], weights=c["weights"])
        elif c["op"] == "window":
            st["bk"].reserve_attend(n_q=c["n_q"])
    return st


# ------------------------------------------------------------------------------------------ passes
def run(state):
    op = state["case"]["op"]
    if own:
        return {"pack": _own_pack, "attend4": _own_attend4, "window": _own_window, "evict4": _own_evict4}[op](state)
    return {"pack": _plain_pack, "attend4": _plain_attend4, "window": _plain_window, "evict4": _plain_evict4}[op](state)


def _own_pack(s):
    s["bk"].pack4(s["K"], s["V"], s["K4"], s["V4"], s["S4"], first=s["first"], length=s["length"])
    s["bk"].unpack4(s["K4"], s["V4"], s["S4"], s["K_out"], s["V_out"], first=s["first"], length=s["length"])
    return {"K": s["K_out"], "V": s["V_out"]}


def _own_attend4(s):
    o, lse = s["bk"].attend4(s["q"], s["K4"], s["V4"], s["S4"], length=s["length"], weights=s["weights"])
    return {"o": o, "lse": lse, "weights": s["weights"]}


def _own_window(s):
    c = s["case"]
    o, lse = s["bk"].attend_window(s["q"], s["K"], s["V"], length=s["length"], window=c["window"],
                                   n_sink=c["n_sink"])
    return {"o": o, "lse": lse}


def _own_evict4(s):
    kept, length = s["bk"].evict4(s["K4"], s["V4"], s["S4"], s["weights"], L=s["length"], budget=s["case"]["budget"],
                                  K4_out=s["K4_out"], V4_out=s["V4_out"], S4_out=s["S4_out"],
                                  weights_out=s["weights_out"])
    return {"K4": s["K4_out"], "V4": s["V4_out"], "S4": s["S4_out"], "weights": s["weights_out"], "kept": kept,
            "length": length}


def _plain_pack(s):
    c = s["case"]
    b, hkv, d, cap, n = c["b"], c["hkv"], c["d"], c["cap"], c["n"]
    # row i of the new rows is row first + i of its cache, where that is below the cache's length
    row = s["first"][..., None].long() + torch.arange(n, device=DEV)
    there = row < s["length"][..., None]
    at = (torch.arange(b * hkv, device=DEV).view(b, hkv, 1) * cap + row)[there]
    for which, (src, codes, back) in enumerate(((s["K"], s["K4"], s["K_out"]), (s["V"], s["V4"], s["V_out"]))):
        code, step, low = _quantise(src[there], torch.float64)
        packed = _words(code, which)
        codes.view(-1, d // 2)[at] = packed
        flat = s["S4"].view(-1, 2, d // GROUP, 2)
        flat[at, which] = torch.stack((step, low), -1).to(torch.float16)
        back[there] = _values(packed, flat[at], which, torch.float32).to(torch.bfloat16)
    return {"K": s["K_out"], "V": s["V_out"]}


def _softmax(q, K, V, seen):
    """Softmax over the keys that `seen` marks, for [.., rows, d] queries: (o, lse, numerators, their sums)."""
    z = (q @ K.transpose(-1, -2) / math.sqrt(q.shape[-1])).masked_fill_(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    safe = torch.where(total > 0, total, torch.ones_like(total))
    return p @ V / safe, (top + torch.log(total))[..., 0], p, safe


def _limits(s):
    """Rows that each query of [b, hkv, group * n_q] sees the causal way."""
    c = s["case"]
    i = torch.arange(c["n_q"], device=DEV).repeat(c["hq"] // c["hkv"])
    return (s["length"][:, :, None] - c["n_q"] + 1 + i)[..., None]


def _plain_attend4(s):
    c = s["case"]
    b, hq, hkv, d, cap, n_q = c["b"], c["hq"], c["hkv"], c["d"], c["cap"], c["n_q"]
    q = s["q"].float().view(b, hkv, hq // hkv * n_q, d)
    seen = torch.arange(cap, device=DEV) < _limits(s)
    o, lse, p, safe = _softmax(q, _values(s["K4"], s["S4"], 0, torch.float32),
                               _values(s["V4"], s["S4"], 1, torch.float32), seen)
    if s["weights"] is not None:
        s["weights"] += (p / safe).sum(-2)
    return {"o": o.to(torch.bfloat16).view(b, hq, n_q, d), "lse": lse.view(b, hq, n_q), "weights": s["weights"]}


def _plain_window(s):
    c = s["case"]
    b, hq, hkv, d, cap, n_q = c["b"], c["hq"], c["hkv"], c["d"], c["cap"], c["n_q"]
    q = s["q"].float().view(b, hkv, hq // hkv * n_q, d)
    j, limit = torch.arange(cap, device=DEV), _limits(s)
    seen = (j < limit) & ((j < c["n_sink"]) | (j >= limit - c["window"]))
    o, lse, _, _ = _softmax(q, s["K"].float(), s["V"].float(), seen)
    return {"o": o.to(torch.bfloat16).view(b, hq, n_q, d), "lse": lse.view(b, hq, n_q)}


def _plain_evict4(s):
    c = s["case"]
    cap, budget = c["cap"], c["budget"]
    L = s["length"][..., None]
    j = torch.arange(cap, device=DEV)
    # the leading rows and the window come first, what is past the length last, ties in index order
    key = torch.where((j < c["n_prefix"]) | (j >= L - c["window"]), math.inf, s["weights"])
    key = torch.where(j < L, key, -math.inf)
    first = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    n = torch.minimum(L, torch.full_like(L, budget))
    there = torch.arange(budget, device=DEV) < n
    first = torch.where(there, first, cap).sort(-1).values
    kept = torch.where(there, first, -1).to(torch.int32)
    at = first.clamp(max=cap - 1)
    for name in ("K4", "V4", "S4"):
        src, dst = s[name].flatten(4), s[name + "_out"].flatten(4)
        rows = at[..., None].expand(*at.shape, src.shape[-1])
        dst[..., :budget, :] = torch.where(there[..., None], torch.gather(src, -2, rows), dst[..., :budget, :])
    s["weights_out"].zero_()
    s["weights_out"][..., :budget] = torch.where(there, torch.gather(s["weights"], -1, at), 0.0)
    return {"K4": s["K4_out"], "V4": s["V4_out"], "S4": s["S4_out"], "weights": s["weights_out"], "kept": kept,
            "length": n[..., 0].to(torch.int32)}


# ------------------------------------------------------------------------------------------ accounting
def _upto(n):
    return n * (n + 1) // 2 if n > 0 else 0


def _visible(length, n_q):
    """Key visits of n_q causal queries at the end of a cache: the sum of max(0, length - n_q + 1 + i)."""
    return _upto(length) - _upto(max(0, length - n_q))


def work(case):
    c = case
    d, row4 = c["d"], 5 * c["d"] // 4  # bytes of a row of K and V in 4 bits, scales included
    lens = _lengths(c.get("layers", 1) * c["b"] * c["hkv"], c["lo"], c["hi"])
    if c["op"] == "pack":
        rows = sum(min(c["n"], n) for n in lens)
        return {"bytes": rows * (4 * d + row4 + row4 + 4 * d) + 8 * len(lens), "flops": 0}
    if c["op"] == "evict4":
        kept = sum(min(n, c["budget"]) for n in lens)
        # the lengths and the weights of the caches read, the kept rows read and written, the new weights, indices
        # and lengths written
        nbytes = sum(4 * n for n in lens) + kept * row4 * 2 + len(lens) * (4 * c["cap_out"] + 4 * c["budget"] + 8)
        return {"bytes": nbytes, "flops": 0}
    group, rows = c["hq"] // c["hkv"], c["b"] * c["hq"] * c["n_q"]
    nbytes = rows * (2 * 2 * d + 4) + 4 * len(lens)
    if c["op"] == "attend4":
        visits = sum(_visible(n, c["n_q"]) for n in lens)
        nbytes += sum(lens) * (row4 + (8 if c["weights"] else 0))
    else:
        w, sink = c["window"], c["n_sink"]
        # a query at limit n sees n rows less those between the first tokens and its window
        visits = sum(_visible(n, c["n_q"]) - _visible(n - w - sink, c["n_q"]) for n in lens)
        unseen = (max(0, n - c["n_q"] + 1 - w - sink) for n in lens)  # by any query
        nbytes += sum(n - x for n, x in zip(lens, unseen)) * 4 * d
    return {"bytes": nbytes, "flops": 4 * d * group * visits}


# ------------------------------------------------------------------------------------------ exact values
def exact(case, seed):
    """From the definitions, in 64 bits, sequence by sequence and head by head."""
    s = prepare(case, seed)
    return {"pack": _exact_pack, "evict4": _exact_evict}.get(case["op"], _exact_attention)(s)


def _exact_pack(s):
    c = s["case"]
    d, n = c["d"], c["n"]
    out = {}
    for name in "KV":
        x = s[name].double()
        y = torch.zeros_like(x)
        for g in range(0, d, GROUP):
            part = x[..., g:g + GROUP]
            lowest, highest = part.min(-1).values, part.max(-1).values
            low = _nearest_half(lowest)
            step = _nearest_half(torch.clamp(highest - low, min=0.0) / 15.0)
            for k in range(GROUP):
                v = part[..., k] - low
                code = torch.zeros_like(v)
                for level in range(15):  # codes above `level`: past the middle, or on it when the next one is even
                    edge = (level + 0.5) * step
                    code += ((v > edge) | ((v == edge) & (level % 2 == 1))) & (step > 0)
                y[..., g + k] = low + step * code
        keep = torch.arange(n, device=DEV) < torch.clamp(s["length"].long(), max=n)[..., None]
        out[name] = y * keep[..., None]
    return out


def _nearest_half(x):
    """The fp16 number nearest to each fp64 x, from the bits of x: 42 bits of its significand go (more below 2^-14),
    half of them added with a tie's last bit in mind."""
    a = x.abs()
    bits = a.view(torch.int64)
    up = bits + ((1 << 41) - 1) + ((bits >> 42) & 1)
    normal = ((up >> 42) << 42).view(torch.float64)
    small = torch.round(a * 2.0 ** 24) / 2.0 ** 24
    y = torch.where(a < 2.0 ** -14, small, normal).clamp(max=TOP)
    return torch.copysign(y, x)


def _codes(words, d, which):
    """Codes of rows of bytes, element by element of the format's definition."""
    out = torch.empty(*words.shape[:-1], d, dtype=torch.float64, device=DEV)
    for e in range(d):
        w, x = (e % 32 // 8 * (d // 32) + e // 32, e % 8) if which == 0 else (e % (d // 8), e // (d // 8))
        out[..., e] = ((words[..., 4 * w + x // 2] >> (4 * (x % 2))) & 15).double()
    return out


def _exact_attention(s):
    c = s["case"]
    b, hq, hkv, d, n_q = c["b"], c["hq"], c["hkv"], c["d"], c["n_q"]
    group = hq // hkv
    o = torch.zeros(b, hq, n_q, d, dtype=torch.float64, device=DEV)
    lse = torch.full((b, hq, n_q), -math.inf, dtype=torch.float64, device=DEV)
    w = s["weights"].double() if s.get("weights") is not None else None
    lens = s["length"].tolist()
    for x in range(b):
        for y in range(hkv):
            n = lens[x][y]
            if n == 0:
                continue
            if c["op"] == "attend4":
                sc = s["S4"][x, y, :n].double().repeat_interleave(GROUP, 2)
                keys = sc[:, 0, :, 1] + sc[:, 0, :, 0] * _codes(s["K4"][x, y, :n], d, 0)
                vals = sc[:, 1, :, 1] + sc[:, 1, :, 0] * _codes(s["V4"][x, y, :n], d, 1)
            else:
                keys, vals = s["K"][x, y, :n].double(), s["V"][x, y, :n].double()
            pos = torch.arange(n, device=DEV)[None, :]
            newest = torch.arange(n_q, device=DEV)[:, None] + (n - n_q)  # position of each query's own row
            hidden = pos > newest
            if c["op"] == "window":
                hidden |= (pos <= newest - c["window"]) & (pos >= c["n_sink"])
            for h in range(y * group, (y + 1) * group):
                z = s["q"][x, h].double() @ keys.T / math.sqrt(d)
                z[hidden] = -math.inf
                t = torch.logsumexp(z, -1)
                prob = torch.exp(z - torch.where(t == -math.inf, 0.0, t)[:, None])
                o[x, h] = prob @ vals
                lse[x, h] = t
                if w is not None:
                    w[x, y, :n] += prob.sum(0)
    out = {"o": o, "lse": lse}
    if c["op"] == "attend4":
        out["weights"] = w
    return out


def _exact_evict(s):
    """Only the accumulators are numbers that could be rounded, and they are moved, not computed: they are taken
    cache by cache in 64 bits; codes and scales are moved bit for bit."""
    c = s["case"]
    budget = c["budget"]
    W = s["weights"].double().cpu().flatten(0, 2)
    out = torch.zeros(W.shape[0], c["cap_out"], dtype=torch.float64)
    for e, n in enumerate(s["length"].flatten().tolist()):
        rows = list(range(n))
        if n > budget:
            w = W[e].tolist()
            inner = rows[c["n_prefix"]:n - c["window"]]
            best = sorted(inner, key=lambda r: (-w[r], r))[:budget - c["n_prefix"] - c["window"]]
            rows = sorted(rows[:c["n_prefix"]] + best + rows[n - c["window"]:])
        out[e, :len(rows)] = W[e, rows]
    return {"K4": None, "V4": None, "S4": None, "weights": out.view(*s["weights_out"].shape), "kept": None,
            "length": None}
