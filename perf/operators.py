"""The attention-and-eviction operators of a decode loop: cases, plain forms and exact values.

Three operators, in the order in which a serving loop uses them:

attend   attention of the newest ``n_q`` queries of every sequence over the sequence's own cache (a length
         per KV head, causal among the new tokens); it also adds each cached key's attention weight,
         summed over the queries and the query heads of its group, to an accumulator.
shared   the same when the batch's sequences continue a long common prefix, whose K and V exist once per
         group of sequences; only the sequences' own rows accumulate weights.
evict    a cache is cut to its budget by accumulated weight: the leading rows, the most recent rows and the
         heaviest others stay, and K, V and the accumulators are compacted into the decode cache.

``run`` is the plain form (elementary torch operations in 32 bits) unless ``own`` is set, and then the
framework's operators.
"""
import math

import torch

own = False

DEV = "cuda"


# ------------------------------------------------------------------------------------------ cases
def _attend(name, b, hq, hkv, d, cap, n_q, lo, hi, weights):
    return {"name": name, "op": "attend", "b": b, "hq": hq, "hkv": hkv, "d": d, "cap": cap, "n_q": n_q, "lo": lo,
            "hi": hi, "weights": weights}


def _shared(name, b, groups, hq, hkv, d, pcap, plo, phi, cap, n_q, lo, hi, weights):
    c = _attend(name, b, hq, hkv, d, cap, n_q, lo, hi, weights)
    c.update({"op": "shared", "groups": groups, "pcap": pcap, "plo": plo, "phi": phi})
    return c


def _evict(name, layers, b, hkv, d, cap, cap_out, lo, hi, budget, n_prefix, window):
    return {"name": name, "op": "evict", "layers": layers, "b": b, "hkv": hkv, "d": d, "cap": cap, "cap_out": cap_out,
            "lo": lo, "hi": hi, "budget": budget, "n_prefix": n_prefix, "window": window}


def listed():
    return [
        # one token of one short sequence, the smallest shape of the workloads: latency only
        _attend("attend_tiny", 1, 4, 2, 64, 1088, 1, 1088, 1088, True),
        # one layer of a decode step between two evictions, Qwen3-4B shape, caches between budget and capacity
        _attend("attend_step", 16, 32, 8, 128, 4224, 1, 4097, 4224, True),
        # one token of a single sequence with the longest cache a context takes: the keys have to be split
        _attend("attend_long", 1, 32, 8, 128, 32768, 1, 32768, 32768, True),
        # batched decoding with very different lengths, empty caches among them, five query heads per group
        _attend("attend_ragged", 8, 40, 8, 128, 8320, 1, 0, 8320, False),
        # a few draft tokens per sequence appended at once, head_dim 64, odd lengths, caches shorter than the draft
        _attend("attend_draft", 7, 32, 8, 64, 2176, 11, 5, 2171, True),
        # a whole prompt: causal attention with the column sums that the first eviction goes by
        _attend("attend_prompt", 1, 32, 8, 128, 4224, 4096, 4096, 4096, True),
        # a few samples of one short prompt, just begun
        _shared("shared_begin", 4, 1, 4, 2, 64, 512, 509, 509, 64, 1, 1, 9, True),
        # sixteen samples of one long prompt in mid-answer: the prefix is read once for all
        _shared("shared_long", 16, 1, 32, 8, 128, 32768, 32768, 32768, 4224, 1, 100, 1200, True),
        # four prompts with sixteen samples each, prompts of odd lengths, five query heads per group
        _shared("shared_groups", 64, 4, 40, 8, 128, 8320, 1031, 8203, 2176, 1, 0, 700, False),
        # one layer of the smallest shape
        _evict("evict_tiny", 1, 1, 2, 64, 1088, 1088, 1088, 1088, 512, 4, 8),
        # eight layers of the Qwen3-4B shape, one period's worth of rows evicted from every cache
        _evict("evict_period", 8, 16, 8, 128, 4224, 4224, 4224, 4224, 4096, 0, 8),
        # long prompts of many lengths cut into a smaller decode cache, some of them already under the budget
        _evict("evict_prompt", 5, 8, 8, 128, 32768, 2176, 1, 32768, 2048, 4, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    d = rng.choice((64, 128))
    hkv = rng.choice((1, 2, 4, 8))
    hq = hkv * rng.choice((1, 2, 4, 5, 7, 8))
    kind = rng.choice(("token", "draft", "prompt", "shared", "evict"))
    if kind == "token":
        b = _log(rng, 1, 32)
        cap = _log(rng, 64, min(32768, 16 * 4224 * 8 // (b * hkv)))
        lo = rng.randint(0, cap)
        c = _attend("", b, hq, hkv, d, cap, 1, lo, rng.randint(max(lo, 1), cap), rng.random() < 0.6)
    elif kind == "draft":
        b = _log(rng, 1, 16)
        cap = _log(rng, 64, min(8320, 16 * 4224 * 8 // (b * hkv)))
        lo = rng.randint(0, cap)
        c = _attend("", b, hq, hkv, d, cap, rng.randint(2, 40), lo, rng.randint(max(lo, 1), cap), rng.random() < 0.6)
    elif kind == "prompt":
        n_q = _log(rng, 65, 4096)
        b = _log(rng, 1, max(1, min(8, 4096 * 4096 * 32 // (n_q * n_q * hq * 4))))
        cap = rng.randint(n_q, min(8320, n_q + 1100))
        while b > 1 and b * hq * n_q * cap > 32 * 4096 * 4224:
            b -= 1
        cap = max(n_q, min(cap, 32 * 4096 * 4224 // (b * hq * n_q)))
        lo = rng.randint(n_q // 2, cap)
        c = _attend("", b, hq, hkv, d, cap, n_q, lo, rng.randint(lo, cap), rng.random() < 0.6)
    elif kind == "shared":
        groups = rng.choice((1, 1, 2, 3))
        b = groups * _log(rng, 2, 48 // groups)
        pcap = _log(rng, 64, min(32768, 16 * 4224 * 8 // (groups * hkv)))
        plo = rng.randint(0, pcap)
        cap = _log(rng, 16, max(16, min(4224, 16 * 4224 * 8 // (b * hkv))))
        lo = rng.randint(0, cap)
        n_q = rng.choice((1, 1, 1, 3))
        c = _shared("", b, groups, hq, hkv, d, pcap, plo, rng.randint(max(plo, 1), pcap), cap, n_q, lo,
                    rng.randint(max(lo, 1), cap), rng.random() < 0.6)
    else:
        layers, b = rng.randint(1, 8), _log(rng, 1, 16)
        cap = _log(rng, 64, min(32768, 8 * 16 * 8 * 4224 // (layers * b * hkv)))
        window = rng.randint(0, min(32, cap // 4))
        n_prefix = rng.choice((0, 1, 4, 7))
        budget = rng.randint(n_prefix + window + 1, cap)
        lo = rng.randint(0, cap)
        c = _evict("", layers, b, hkv, d, cap, rng.randint(budget, cap), lo, rng.randint(lo, cap), budget, n_prefix,
                   window)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _lengths(n, lo, hi):
    """n lengths spread evenly over lo..hi, both ends among them, in a fixed scattered order: the work of a case
    does not depend on the seed."""
    step = next(s for s in range(max(1, int(n * 0.618)), 2 * n + 2) if math.gcd(s, n) == 1)
    return [hi if n == 1 else lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _randn(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype)


def _cache(gen, b, hkv, cap, d):
    """K and V of one layer: keys with a mean of their own per head, as the workloads' have."""
    K, V = _randn(gen, b, hkv, cap, d), _randn(gen, b, hkv, cap, d)
    K += 0.5 * _randn(gen, 1, hkv, 1, d)
    return K, V


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    c, st = case, {"case": case}
    b, hkv, d, cap = c["b"], c["hkv"], c["d"], c["cap"]
    if c["op"] == "evict":
        layers, out = c["layers"], c["cap_out"]
        st["K"] = _randn(gen, layers, b, hkv, cap, d)
        st["V"] = _randn(gen, layers, b, hkv, cap, d)
        # accumulated weights: heavy-tailed, with many equal small values (rows seen by few queries)
        w = torch.exp(1.5 * _randn(gen, layers, b, hkv, cap, dtype=torch.float32) - 3)
        st["weights"] = torch.where(w < 0.03, torch.round(w * 256) / 256, w)
        st["L"] = torch.tensor(_lengths(layers * b * hkv, c["lo"], c["hi"]), dtype=torch.int32,
                               device=DEV).view(layers, b, hkv)
        st["K_out"], st["V_out"] = (torch.zeros(layers, b, hkv, out, d, dtype=torch.bfloat16, device=DEV) for _ in "KV")
        st["weights_out"] = torch.zeros(layers, b, hkv, out, device=DEV)
    else:
        st["K"], st["V"] = _cache(gen, b, hkv, cap, d)
        st["q"] = _randn(gen, b, c["hq"], c["n_q"], d) * 2
        st["length"] = torch.tensor(_lengths(b * hkv, c["lo"], c["hi"]), dtype=torch.int32, device=DEV).view(b, hkv)
        st["weights"] = None
        if c["weights"]:
            st["weights"] = torch.rand(b, hkv, cap, generator=gen, device=DEV)
        if c["op"] == "shared":
            st["Kp"], st["Vp"] = _cache(gen, c["groups"], hkv, c["pcap"], d)
            st["prefix_len"] = torch.tensor(_lengths(c["groups"], c["plo"], c["phi"]), dtype=torch.int32, device=DEV)
    if own:
        from paper_2609_04971_gb300 import bkv
        shape = dict(n_layers=c.get("layers", 1), batch=b, n_q_heads=c.get("hq", hkv), n_kv_heads=hkv, head_dim=d,
                     n_beacons=0 if c.get("window", 1) else 1, window=c.get("window", 1), capacity=cap,
                     n_prefix=c.get("n_prefix", 0))
        st["bk"] = bkv.BeaconKV(**shape)
        if c["op"] != "evict":
            st["bk"].reserve_attend(n_q=c["n_q"], n_groups=c.get("groups", 0), weights=c["weights"])
    return st


# ------------------------------------------------------------------------------------------ passes
def run(state):
    c = state["case"]
    if own:
        return {"attend": _own_attend, "shared": _own_shared, "evict": _own_evict}[c["op"]](state)
    return {"attend": _plain_attend, "shared": _plain_attend, "evict": _plain_evict}[c["op"]](state)


def _own_attend(s):
    o, lse = s["bk"].attend(s["q"], s["K"], s["V"], length=s["length"], weights=s["weights"])
    return {"o": o, "lse": lse, "weights": s["weights"]}


def _own_shared(s):
    o, lse = s["bk"].attend_shared(s["q"], s["Kp"], s["Vp"], s["K"], s["V"], prefix_len=s["prefix_len"],
                                   length=s["length"], weights=s["weights"])
    return {"o": o, "lse": lse, "weights": s["weights"]}


def _own_evict(s):
    c = s["case"]
    kept, length = s["bk"].evict(s["K"], s["V"], s["weights"], L=s["L"], budget=c["budget"], K_out=s["K_out"],
                                 V_out=s["V_out"], weights_out=s["weights_out"])
    return {"K": s["K_out"], "V": s["V_out"], "weights": s["weights_out"], "kept": kept, "length": length}


def _plain_attend(s):
    c = s["case"]
    b, hq, hkv, d, cap, n_q = c["b"], c["hq"], c["hkv"], c["d"], c["cap"], c["n_q"]
    rows = hq // hkv * n_q
    q = s["q"].float().view(b, hkv, rows, d)
    K, V = s["K"].float(), s["V"].float()
    scale = 1.0 / math.sqrt(d)
    # query i of n_q sees the rows below length - n_q + 1 + i
    i = torch.arange(n_q, device=DEV).repeat(hq // hkv)
    limit = s["length"][:, :, None] - n_q + 1 + i
    masked = torch.arange(cap, device=DEV) >= limit[..., None]
    logits = (q @ K.transpose(-1, -2) * scale).masked_fill_(masked, -math.inf)
    top = logits.amax(-1, keepdim=True)
    if c["op"] == "shared":
        g, m, pcap = c["groups"], b // c["groups"], c["pcap"]
        qp = q.view(g, m, hkv, rows, d).transpose(1, 2).reshape(g, hkv, m * rows, d)
        beyond = torch.arange(pcap, device=DEV) >= s["prefix_len"][:, None, None, None]
        plogits = (qp @ s["Kp"].float().transpose(-1, -2) * scale).masked_fill_(beyond, -math.inf)
        ptop = plogits.amax(-1, keepdim=True)
        ptop = ptop.view(g, hkv, m, rows, 1).transpose(1, 2).reshape(b, hkv, rows, 1)
        top = torch.maximum(top, ptop)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    mixed = p @ V
    if c["op"] == "shared":
        ref = top.view(g, m, hkv, rows, 1).transpose(1, 2).reshape(g, hkv, m * rows, 1)
        pp = torch.exp(plogits - ref)
        ptotal, pmixed = pp.sum(-1, keepdim=True), pp @ s["Vp"].float()
        total = total + ptotal.view(g, hkv, m, rows, 1).transpose(1, 2).reshape(b, hkv, rows, 1)
        mixed = mixed + pmixed.view(g, hkv, m, rows, d).transpose(1, 2).reshape(b, hkv, rows, d)
    safe = torch.where(total > 0, total, torch.ones_like(total))
    o = (mixed / safe).to(torch.bfloat16).view(b, hq, n_q, d)
    lse = (top + torch.log(total)).view(b, hq, n_q)
    if s["weights"] is not None:
        s["weights"] += (p / safe).sum(-2)
    return {"o": o, "lse": lse, "weights": s["weights"]}


def _plain_evict(s):
    c = s["case"]
    cap, out, budget = c["cap"], c["cap_out"], c["budget"]
    L = s["L"][..., None]
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
    rows = at[..., None].expand(*at.shape, c["d"])
    for src, dst in ((s["K"], s["K_out"]), (s["V"], s["V_out"])):
        dst[..., :budget, :] = torch.where(there[..., None], torch.gather(src, -2, rows), dst[..., :budget, :])
    s["weights_out"].zero_()
    s["weights_out"][..., :budget] = torch.where(there, torch.gather(s["weights"], -1, at), 0.0)
    return {"K": s["K_out"], "V": s["V_out"], "weights": s["weights_out"], "kept": kept,
            "length": n[..., 0].to(torch.int32)}


# ------------------------------------------------------------------------------------------ accounting
def _visible(length, n_q):
    """Key visits of n_q causal queries at the end of a cache: the sum of max(0, length - n_q + 1 + i)."""
    hi, lo = length, max(0, length - n_q)
    return (hi * (hi + 1) - lo * (lo + 1)) // 2


def work(case):
    c = case
    d = c["d"]
    if c["op"] == "evict":
        lens = _lengths(c["layers"] * c["b"] * c["hkv"], c["lo"], c["hi"])
        kept = sum(min(n, c["budget"]) for n in lens)
        # the lengths and the weights of the caches read, the kept rows of K and V read and written, the new
        # weights, indices and lengths written
        nbytes = sum(4 * n for n in lens) + kept * d * 2 * 4 + len(lens) * (4 * c["cap_out"] + 4 * c["budget"] + 8)
        return {"bytes": nbytes, "flops": 0}
    lens = _lengths(c["b"] * c["hkv"], c["lo"], c["hi"])
    group, rows = c["hq"] // c["hkv"], c["b"] * c["hq"] * c["n_q"]
    visits = group * sum(_visible(n, c["n_q"]) for n in lens)
    nbytes = rows * (2 * 2 * d + 4) + sum(lens) * 2 * 2 * d + 4 * len(lens)
    if c["weights"]:
        nbytes += 8 * sum(lens)
    if c["op"] == "shared":
        plens = _lengths(c["groups"], c["plo"], c["phi"])
        visits += sum(plens) * (c["b"] // c["groups"]) * c["hq"] * c["n_q"]
        nbytes += sum(plens) * c["hkv"] * 2 * 2 * d + 4 * len(plens)
    return {"bytes": nbytes, "flops": 4 * d * visits}


# ------------------------------------------------------------------------------------------ exact values
def exact(case, seed):
    """From the definitions, in 64 bits, sequence by sequence and head by head."""
    s = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(s)
    c = case
    b, hq, hkv, d, n_q = c["b"], c["hq"], c["hkv"], c["d"], c["n_q"]
    group = hq // hkv
    o = torch.zeros(b, hq, n_q, d, dtype=torch.float64, device=DEV)
    lse = torch.full((b, hq, n_q), -math.inf, dtype=torch.float64, device=DEV)
    w = None if s["weights"] is None else s["weights"].double()
    lens = s["length"].tolist()
    plens = s["prefix_len"].tolist() if c["op"] == "shared" else None
    for x in range(b):
        for y in range(hkv):
            n, P = lens[x][y], 0
            keys, vals = s["K"][x, y, :n].double(), s["V"][x, y, :n].double()
            if plens is not None:
                grp = x // (b // c["groups"])
                P = plens[grp]
                keys = torch.cat([s["Kp"][grp, y, :P].double(), keys])
                vals = torch.cat([s["Vp"][grp, y, :P].double(), vals])
            if P + n == 0:
                continue
            for h in range(y * group, (y + 1) * group):
                z = s["q"][x, h].double() @ keys.T / math.sqrt(d)
                pos = torch.arange(P + n, device=DEV)
                newest = torch.arange(n_q, device=DEV)[:, None] + (P + n - n_q)
                z[(pos[None, :] >= P) & (pos[None, :] > newest)] = -math.inf
                t = torch.logsumexp(z, -1)
                prob = torch.exp(z - torch.where(t == -math.inf, 0.0, t)[:, None])
                o[x, h] = prob @ vals
                lse[x, h] = t
                if w is not None:
                    w[x, y, :n] += prob[:, P:].sum(0)
    return {"o": o, "lse": lse, "weights": w}


def _exact_evict(s):
    """Only the accumulators are numbers that could be rounded, and they are moved, not computed: they are taken
    cache by cache in 64 bits; K and V are moved bit for bit."""
    c = s["case"]
    budget = c["budget"]
    W = s["weights"].double().cpu().flatten(0, 2)
    out = torch.zeros(W.shape[0], c["cap_out"], dtype=torch.float64)
    for e, n in enumerate(s["L"].flatten().tolist()):
        rows = list(range(n))
        if n > budget:
            w = W[e].tolist()
            inner = rows[c["n_prefix"]:n - c["window"]]
            best = sorted(inner, key=lambda r: (-w[r], r))[:budget - c["n_prefix"] - c["window"]]
            rows = sorted(rows[:c["n_prefix"]] + best + rows[n - c["window"]:])
        out[e, :len(rows)] = W[e, rows]
    return {"K": None, "V": None, "weights": out.view(*s["weights_out"].shape), "kept": None, "length": None}
