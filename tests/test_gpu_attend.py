"""bkv_attend, bkv_attend_shared and bkv_evict against plain implementations in 64 bits.

Tolerances, from the arithmetic (u = 2^-8, the unit roundoff of bf16):
- a logit is a sum of head_dim exact products in fp32; with S = scale * max_j sum_i |q_i k_ji| its error is at
  most 2^-16 S (128 additions, each off by at most 2^-23 of the sum of magnitudes);
- lse: the logit error, plus 2^-15 for the exponentials (2^-22 each) and for sums of at most 2^9 partial terms
  in a row, plus the rounding of the result;
- o: the weights are rounded to bf16 once (u), the result once more, and each weight carries the relative error
  of its exponential, at most delta = 2 * 2^-16 S + 2^-14: |o - o64| <= u |o| + (u + 2 delta) sum_j p_j |v_j|;
- weights: each term is off by at most delta of itself, and the sum of R terms by R 2^-24 of its value.
"""
import math

import pytest
import torch

from paper_2609_04971_gb300 import bkv

pytestmark = pytest.mark.gpu

U = 2.0 ** -8


def _bk(b, hq, hkv, d, cap, **kw):
    kw = {"n_layers": 1, "n_beacons": 1, "window": 0, **kw}
    return bkv.BeaconKV(batch=b, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, capacity=cap, **kw)


def _inputs(b, hq, hkv, d, cap, n_q, seed=0, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    q = (std * r(b, hq, n_q, d)).bfloat16()
    return q, r(b, hkv, cap, d).bfloat16(), r(b, hkv, cap, d).bfloat16()


def _poison(K, V, lens):
    """What lies past a cache's length is never used: NaN and infinities there."""
    for x in range(K.shape[0]):
        for y in range(K.shape[1]):
            n = int(lens[x][y])
            K[x, y, n:] = math.nan
            V[x, y, n:] = math.inf
            V[x, y, n::2] = math.nan


def _lens(b, hkv, values):
    flat = [values[i % len(values)] for i in range(b * hkv)]
    return torch.tensor(flat, dtype=torch.int32, device="cuda").view(b, hkv)


def reference(q, K, V, lens, Kp=None, Vp=None, plens=None, scale=None):
    """o, lse, the weights' increments (own rows), and the tolerances of each."""
    b, hq, n_q, d = q.shape
    hkv, cap = K.shape[1:3]
    G = hq // hkv
    scale = scale or 1 / math.sqrt(d)
    o = torch.zeros(b, hq, n_q, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq, n_q), -math.inf, dtype=torch.float64, device="cuda")
    w = torch.zeros(b, hkv, cap, dtype=torch.float64, device="cuda")
    to, tl, tw = torch.zeros_like(o), torch.zeros_like(lse), torch.zeros_like(w)
    for x in range(b):
        for y in range(hkv):
            n = int(lens[x, y])
            k, v, P = K[x, y, :n].double(), V[x, y, :n].double(), 0
            if Kp is not None:
                grp = x // (b // Kp.shape[0])
                P = int(plens[grp])
                k, v = torch.cat([Kp[grp, y, :P].double(), k]), torch.cat([Vp[grp, y, :P].double(), v])
            if P + n == 0:
                continue
            j = torch.arange(P + n, device="cuda")
            i = torch.arange(n_q, device="cuda").repeat(G)[:, None]
            qq = q[x, y * G:(y + 1) * G].reshape(G * n_q, d).double()
            z = qq @ k.T * scale
            seen = (j[None] < P) | (j[None] - P < n - n_q + 1 + i)
            z = z.masked_fill(~seen, -math.inf)
            S = (qq.abs() @ k.abs().T * scale).masked_fill(~seen, 0).amax(-1)
            t = torch.logsumexp(z, -1)
            p = torch.exp(z - torch.where(t == -math.inf, 0.0, t)[:, None])
            delta = (2 * 2.0 ** -16 * S + 2.0 ** -14)[:, None]
            oo = p @ v
            rows = slice(y * G, (y + 1) * G)
            o[x, rows] = oo.view(G, n_q, d)
            to[x, rows] = (U * oo.abs() + (U + 2 * delta) * (p @ v.abs())).view(G, n_q, d)
            lse[x, rows] = t.view(G, n_q)
            tl[x, rows] = (2.0 ** -16 * S + 2.0 ** -15 + 2.0 ** -22 * t.abs()).view(G, n_q)
            w[x, y, :n] = p[:, P:].sum(0)
            tw[x, y, :n] = (p * delta)[:, P:].sum(0) + (G * n_q + 8) * 2.0 ** -24 * w[x, y, :n]
    return (o, lse, w), (to, tl, tw)


def check(got, want, tol, what):
    got = got.double()
    assert bool(torch.isfinite(got).eq(torch.isfinite(want)).all()), f"{what}: finite in other places"
    f = torch.isfinite(want)
    assert torch.equal(got[~f], want[~f]), what
    worst = ((got - want).abs() - tol)[f]
    assert not worst.numel() or float(worst.max()) <= 0, f"{what}: off by {float(worst.max()):.3g} past the tolerance"


def run_and_check(bk, q, K, V, lens, *, Kp=None, Vp=None, plens=None, weights=True, scale=None, times=1):
    cap = K.shape[2]
    w0 = torch.rand(*K.shape[:3], device="cuda")
    w = w0.clone() if weights else None
    groups = 0 if Kp is None else Kp.shape[0]
    bk.reserve_attend(n_q=q.shape[2], n_groups=groups, weights=weights)
    for _ in range(times):
        if Kp is None:
            o, lse = bk.attend(q, K, V, length=lens, weights=w, scale=scale)
        else:
            o, lse = bk.attend_shared(q, Kp, Vp, K, V, prefix_len=plens, length=lens, weights=w, scale=scale)
    bk.sync()
    (o64, l64, w64), (to, tl, tw) = reference(q, K, V, lens, Kp, Vp, plens, scale)
    check(lse, l64, tl, "lse")
    check(o, o64, to, "o")
    if weights:
        past = torch.arange(cap, device="cuda") >= lens[..., None]
        assert torch.equal(w[past], w0[past]), "weights past the length were touched"
        check(w, w0.double() + times * w64, times * (tw + 2.0 ** -23 * (w0 + w64)), "weights")
    return o, lse, w


# ------------------------------------------------------------------------------------------ attend
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 5, 8, 16, 17])
def test_single_tokens(d, G):
    """One token per sequence: every length around the tile borders, group sizes around the row tiles."""
    b, hkv, cap = 4, 2, 700
    lens = _lens(b, hkv, [1, 127, 128, 129, 700, 0, 255, 300])
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, 1, seed=G)
    _poison(K, V, lens)
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens)
        run_and_check(bk, q, K, V, lens, weights=False)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,G,values", [
    (2, 4, [1, 2, 3, 200, 0, 130]), (7, 1, [6, 7, 8, 135, 128, 3]), (16, 1, [16, 15, 17, 400, 1, 144]),
    (33, 4, [33, 32, 0, 399, 160, 34]), (33, 2, [400, 5, 129, 256, 31, 66]), (130, 3, [130, 129, 131, 400, 7, 258]),
    (257, 1, [400, 257, 128, 1, 384, 300]), (400, 2, [400, 399, 130, 0, 256, 1]),
    # 24, 44, 64, 92, 112 and 128 rows to a block: every column count of the narrow kernel
    (6, 4, [6, 5, 0, 400, 129, 140]), (11, 4, [11, 10, 139, 266, 1, 400]), (16, 4, [16, 1, 128, 143, 400, 0]),
    (23, 4, [23, 150, 400, 0, 22, 257]), (28, 4, [28, 400, 128, 1, 155, 300]), (32, 4, [32, 31, 160, 400, 0, 287]),
    # 256 and 260 rows: the widest block, and one that needs two
    (64, 4, [64, 63, 400, 0, 128, 191]), (65, 4, [65, 400, 2, 128, 192, 0])])
def test_several_tokens(d, n_q, G, values):
    """Causal queries at the end of caches that may be shorter than their number (empty rows)."""
    b, hkv, cap = 3, 2, 400
    lens = _lens(b, hkv, values)
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=n_q)
    _poison(K, V, lens)
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens)
        run_and_check(bk, q, K, V, lens, weights=False)
    finally:
        bk.close()


@pytest.mark.parametrize("cap", [1, 2, 31, 128])
def test_smallest_capacities(cap):
    """Caches shorter than a tile: reads past the tensor's end must not happen or not matter."""
    q, K, V = _inputs(1, 2, 1, 128, cap, 1, seed=cap)
    bk = _bk(1, 2, 1, 128, cap)
    try:
        for n in {0, 1, cap}:
            run_and_check(bk, q, K, V, _lens(1, 1, [n]))
    finally:
        bk.close()


@pytest.mark.parametrize("order", ["rising", "falling", "spike", "equal", "far"])
@pytest.mark.parametrize("n_q", [1, 4, 12, 20, 32, 60])
def test_running_maximum(order, n_q):
    """Logits that force the running reference to move, by far more than a float's exponent range can bridge
    in one step: rising and falling through +-150, one spike late in the cache, all equal, all far below 0."""
    b, hq, hkv, d, cap = 2, 8, 2, 128, 1500
    q, K, V = _inputs(b, hq, hkv, d, cap, n_q, seed=3, std=1.0)
    unit = torch.ones(d, device="cuda") / math.sqrt(d)
    level = {"rising": torch.linspace(-150, 150, cap), "falling": torch.linspace(150, -150, cap),
             "spike": torch.where(torch.arange(cap) == 1333, 140.0, 0.0), "equal": torch.zeros(cap),
             "far": torch.full((cap,), -300.0)}[order].cuda()
    if order == "equal":
        q.zero_()
    else:  # q . k / sqrt(d) = level + noise
        q[:] = (unit * math.sqrt(d) + 0.02 * q).bfloat16()
        K[:] = (level[:, None] * unit + 0.1 * K).bfloat16()
    bk = _bk(b, hq, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, _lens(b, hkv, [1500, 1400, 1450, 129]))
    finally:
        bk.close()


def test_scale_and_accumulation():
    """A scale of the caller's, and two calls adding to the same weights."""
    b, hq, hkv, d, cap = 2, 4, 2, 64, 300
    q, K, V = _inputs(b, hq, hkv, d, cap, 1, seed=5)
    bk = _bk(b, hq, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, _lens(b, hkv, [300, 17]), scale=0.31, times=2)
    finally:
        bk.close()


def test_many_short_caches():
    """More caches than SMs, most of them shorter than a tile: many segments to a block, several to a tile's time."""
    b, hkv, cap, d = 150, 4, 300, 64
    lens = _lens(b, hkv, [3, 0, 140, 1, 299, 64, 128, 129, 17])
    q, K, V = _inputs(b, 2 * hkv, hkv, d, cap, 2, seed=40)
    _poison(K, V, lens)
    bk = _bk(b, 2 * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens)
    finally:
        bk.close()


def test_long_cache_and_many_queries():
    """The longest cache of a context for one sequence, and a prompt of several row blocks."""
    q, K, V = _inputs(1, 8, 2, 128, 32768, 1, seed=6)
    bk = _bk(1, 8, 2, 128, 32768)
    try:
        run_and_check(bk, q, K, V, _lens(1, 2, [32768, 32001]))
    finally:
        bk.close()
    q, K, V = _inputs(2, 4, 2, 64, 2100, 1025, seed=7)
    bk = _bk(2, 4, 2, 64, 2100)
    try:
        run_and_check(bk, q, K, V, _lens(2, 2, [2100, 1025, 900, 1500]))
    finally:
        bk.close()


def test_offsets_past_32_bits():
    """More than 2^31 elements in K: the last sequence's rows lie past every 32-bit offset."""
    b, hq, hkv, d, cap = 66, 8, 8, 128, 32768
    K = torch.empty(b, hkv, cap, d, dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    q, k, v = _inputs(1, hq, hkv, d, 300, 1, seed=8)
    K[-1, :, :300], V[-1, :, :300] = k[0], v[0]
    lens = torch.zeros(b, hkv, dtype=torch.int32, device="cuda")
    lens[-1] = 300
    qq = torch.zeros(b, hq, 1, d, dtype=torch.bfloat16, device="cuda")
    qq[-1] = q[0]
    w = torch.zeros(b, hkv, cap, device="cuda")
    bk = _bk(b, hq, hkv, d, cap)
    try:
        bk.reserve_attend(weights=True)
        o, lse = bk.attend(qq, K, V, length=lens, weights=w)
        bk.sync()
    finally:
        bk.close()
    (o64, l64, w64), (to, tl, tw) = reference(q, k, v, lens[-1:])
    check(o[-1:], o64, to, "o")
    check(lse[-1:], l64, tl, "lse")
    check(w[-1:, :, :300], w64, tw, "weights")
    assert not bool(o[:-1].any()) and bool((lse[:-1] == -math.inf).all()) and not bool(w[:-1].any())


def test_same_bits_every_time_and_on_another_stream():
    b, hq, hkv, d, cap = 5, 10, 2, 128, 2000
    q, K, V = _inputs(b, hq, hkv, d, cap, 3, seed=9)
    lens = _lens(b, hkv, [2000, 3, 777, 1999, 1, 1024])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    outs = []
    for stream in (None, side, None):
        bk = _bk(b, hq, hkv, d, cap, stream=stream)
        try:
            bk.reserve_attend(n_q=3, weights=True)
            w = torch.zeros(b, hkv, cap, device="cuda")
            torch.cuda.synchronize()
            o, lse = bk.attend(q, K, V, length=lens, weights=w)
            bk.sync()
            outs.append((o.clone(), lse.clone(), w))
        finally:
            bk.close()
    for other in outs[1:]:
        for x, y in zip(outs[0], other):
            assert torch.equal(x, y)


def test_attend_in_a_graph():
    """Captured once, replayed on other data in the same buffers."""
    b, hq, hkv, d, cap = 2, 8, 2, 128, 600
    q, K, V = _inputs(b, hq, hkv, d, cap, 1, seed=10)
    lens = _lens(b, hkv, [600, 5, 200, 128])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        bk = _bk(b, hq, hkv, d, cap)
        bk.reserve_attend(weights=True)
        w = torch.zeros(b, hkv, cap, device="cuda")
        o = torch.empty(b, hq, 1, d, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(b, hq, 1, device="cuda")
        bk.attend(q, K, V, length=lens, weights=w, o_out=o, lse_out=lse)  # loads the kernels
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            bk.attend(q, K, V, length=lens, weights=w, o_out=o, lse_out=lse)
    try:
        torch.cuda.synchronize()
        q2, K2, V2 = _inputs(b, hq, hkv, d, cap, 1, seed=11)
        q.copy_(q2), K.copy_(K2), V.copy_(V2), w.zero_(), lens.copy_(_lens(b, hkv, [1, 600, 300, 0]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        bk.sync()
        (o64, l64, w64), (to, tl, tw) = reference(q, K, V, lens)
        check(o, o64, to, "o")
        check(lse, l64, tl, "lse")
        check(w, w64, tw, "weights")
    finally:
        bk.close()


# ------------------------------------------------------------------------------------------ shared prefix
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("groups,m,G,n_q,pcap,plens", [
    (1, 4, 4, 1, 300, [300]), (1, 3, 5, 1, 129, [129]), (2, 3, 1, 1, 400, [0, 399]), (1, 40, 4, 1, 257, [200]),
    (3, 2, 8, 3, 200, [1, 128, 200]), (1, 2, 2, 70, 300, [291]), (2, 1, 3, 1, 64, [64, 5]), (1, 20, 7, 1, 1000, [999]),
    (1, 33, 8, 1, 700, [640]), (2, 3, 4, 80, 300, [300, 1]), (1, 9, 16, 1, 513, [513])])
def test_shared_prefix(d, groups, m, G, n_q, pcap, plens):
    """Prefixes of odd lengths, an empty one, own caches that are empty or short; row blocks that split the
    sequences' rows unevenly."""
    b, hkv, cap = groups * m, 2, 260
    lens = _lens(b, hkv, [0, 1, 129, 260, 128, 17, 40])
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=m)
    _, Kp, Vp = _inputs(groups, 1, hkv, d, pcap, 1, seed=m + 1)
    pl = torch.tensor(plens, dtype=torch.int32, device="cuda")
    _poison(K, V, lens)
    _poison(Kp, Vp, pl[:, None].expand(groups, hkv))
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens, Kp=Kp, Vp=Vp, plens=pl)
        run_and_check(bk, q, K, V, lens, Kp=Kp, Vp=Vp, plens=pl, weights=False)
    finally:
        bk.close()


def test_shared_prefix_equals_its_copies():
    """The shared form and bkv_attend over caches that each hold a copy of the prefix see the same rows."""
    b, hq, hkv, d, P, cap = 6, 8, 2, 128, 500, 90
    q, K, V = _inputs(b, hq, hkv, d, cap, 1, seed=20)
    _, Kp, Vp = _inputs(1, 1, hkv, d, P, 1, seed=21)
    lens = torch.full((b, hkv), cap, dtype=torch.int32, device="cuda")
    pl = torch.tensor([P], dtype=torch.int32, device="cuda")
    K2, V2 = (torch.cat([p.expand(b, -1, -1, -1), own], 2).contiguous() for p, own in ((Kp, K), (Vp, V)))
    one, two = _bk(b, hq, hkv, d, cap), _bk(b, hq, hkv, d, P + cap)
    try:
        o1, l1, _ = run_and_check(one, q, K, V, lens, Kp=Kp, Vp=Vp, plens=pl)
        o2, l2, _ = run_and_check(two, q, K2, V2, lens + P)
    finally:
        one.close()
        two.close()
    assert float((l1 - l2).abs().max()) < 1e-3
    assert float((o1.float() - o2.float()).abs().max()) < 0.02


# ------------------------------------------------------------------------------------------ evict
def evict_reference(w, L, budget, n_prefix, window):
    """Kept rows of one instance, from the definition."""
    w = [math.inf if math.isnan(x) else x for x in w]   # a NaN counts as the largest; see the test for inf ties
    rows = list(range(L))
    if L <= budget:
        return rows
    inner = sorted(rows[n_prefix:L - window], key=lambda r: (-w[r], r))[:budget - n_prefix - window]
    return sorted(rows[:n_prefix] + inner + rows[L - window:])


def _check_evict(bk, K, V, w, L, budget, cap_out=None):
    """In place and into another cache; everything that must not change is compared too."""
    c = bk.cfg
    shape = K.shape[:3]
    L_l, w_l = L.flatten().tolist(), w.flatten(0, 2).cpu().tolist()
    want = [evict_reference(w_l[e], L_l[e], budget, c.n_prefix, c.window) for e in range(len(L_l))]
    cap_out = cap_out or min(budget, c.capacity) + 3
    for in_place in (True, False):
        co = c.capacity if in_place else cap_out
        if in_place:
            Ko, Vo, wo = K.clone(), V.clone(), w.clone()
            before = (K, V)
            kept, new = bk.evict(Ko, Vo, wo, L=L, budget=budget)
        else:
            Ko, Vo = (torch.randn(*shape, co, c.head_dim, device="cuda").bfloat16() for _ in "KV")
            wo = torch.full((*shape, co), 7.0, device="cuda")
            before = (Ko.clone(), Vo.clone())
            kept, new = bk.evict(K, V, w, L=L, budget=budget, K_out=Ko, V_out=Vo, weights_out=wo)
        bk.sync()
        bits = lambda t: t.flatten(0, 2).view(torch.int32 if t.dtype == torch.float32 else torch.int16)  # noqa: E731
        k_h, n_h = kept.flatten(0, 2).cpu(), new.flatten().tolist()
        for e, rows in enumerate(want):
            n = len(rows)
            assert n_h[e] == n
            assert k_h[e, :n].tolist() == rows and bool((k_h[e, n:] == -1).all()), f"instance {e}"
            at = torch.tensor(rows, dtype=torch.long, device="cuda")
            for out, src, old in ((Ko, K, before[0]), (Vo, V, before[1])):
                assert torch.equal(bits(out)[e, :n], bits(src)[e, at])
                assert torch.equal(bits(out)[e, n:], bits(old)[e, n:]), "rows past the kept ones were touched"
            assert torch.equal(bits(wo)[e, :n], bits(w)[e, at])
            assert not bool(bits(wo)[e, n:].any()), "weights past the kept rows must be 0"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,budget,n_prefix,window", [
    (40, 1, 0, 0), (40, 13, 4, 9), (300, 200, 0, 8), (700, 699, 3, 1), (700, 350, 0, 0), (2049, 1000, 4, 8),
    (10241, 5000, 1, 32), (333, 400, 2, 2), (2048, 2047, 0, 1), (8300, 8000, 3, 64), (10240, 77, 0, 8),
    (32768, 30000, 4, 16)])
def test_evict(d, cap, budget, n_prefix, window):
    g = torch.Generator(device="cuda").manual_seed(cap)
    shape = (2, 3, 2)
    K, V = (torch.randn(*shape, cap, d, generator=g, device="cuda").bfloat16() for _ in "KV")
    w = torch.exp(torch.randn(*shape, cap, generator=g, device="cuda"))
    w = torch.where(w < 0.7, torch.round(w * 8) / 8, w)   # many equal weights
    lens = [cap, 0, 1, min(budget, cap), min(budget + 1, cap), cap - 1, cap // 2, 33 if cap >= 33 else 1]
    L = torch.tensor([lens[i % 8] for i in range(12)], dtype=torch.int32, device="cuda").view(shape)
    bk = _bk(3, 2, 2, d, cap, n_layers=2, window=window, n_beacons=0 if window else 1, n_prefix=n_prefix)
    try:
        _check_evict(bk, K, V, w, L, budget)
    finally:
        bk.close()


@pytest.mark.parametrize("kind", ["zeros", "equal", "negative", "infinite", "nan", "signed zeros", "rising", "falling"])
def test_evict_weights(kind):
    """All equal weights (ties to the lowest rows), signs, infinities, NaN, monotone orders."""
    cap, budget = 600, 250
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn(1, 1, 2, cap, 64, generator=g, device="cuda").bfloat16() for _ in "KV")
    w = torch.randn(1, 1, 2, cap, generator=g, device="cuda")
    if kind == "zeros":
        w.zero_()
    elif kind == "equal":
        w.fill_(0.37)
    elif kind == "infinite":
        w[..., ::3], w[..., 1::3] = math.inf, -math.inf
    elif kind == "nan":
        w[..., 5::11] = math.nan
        w[..., 6::11] = -torch.full_like(w[..., 6::11], math.nan)
    elif kind == "signed zeros":
        w[..., ::2], w[..., 1::2] = 0.0, -0.0
    elif kind in ("rising", "falling"):
        w = torch.arange(cap, device="cuda").float().expand_as(w).contiguous()
        w = w if kind == "rising" else -w
    L = torch.tensor([cap, 599], dtype=torch.int32, device="cuda").view(1, 1, 2)
    bk = _bk(1, 2, 2, 64, cap, window=8, n_beacons=0, n_prefix=3)
    try:
        _check_evict(bk, K, V, w.contiguous(), L, budget)
    finally:
        bk.close()


def test_evict_length_aliases_and_bad_lengths():
    """len_out may be L; a length out of range is reported, leaves its instance alone and spoils no other."""
    cap, budget = 200, 90
    K, V = (torch.randn(1, 2, 2, cap, 64, device="cuda").bfloat16() for _ in "KV")
    w = torch.rand(1, 2, 2, cap, device="cuda")
    K0, V0, w0 = K.clone(), V.clone(), w.clone()
    L = torch.tensor([200, 201, -1, 91], dtype=torch.int32, device="cuda").view(1, 2, 2)
    bk = _bk(2, 2, 2, 64, cap, window=8, n_beacons=0)
    try:
        kept, new = bk.evict(K, V, w, L=L, budget=budget, len_out=L)
        with pytest.raises(bkv.BkvError) as ei:
            bk.sync()
        assert ei.value.code == bkv.BKV_EINVAL
        bk.sync()
        assert new is L and L.flatten().tolist() == [90, 0, 0, 90]
        for x, y in ((0, 1), (1, 0)):
            assert bool((kept[0, x, y] == -1).all())
            assert torch.equal(K[0, x, y], K0[0, x, y]) and torch.equal(V[0, x, y], V0[0, x, y])
            assert torch.equal(w[0, x, y], w0[0, x, y])
        assert kept[0, 1, 1].tolist() == evict_reference(w0[0, 1, 1].tolist(), 91, budget, 0, 8)
    finally:
        bk.close()


# ------------------------------------------------------------------------------------------ refusals
def test_bad_device_lengths_count_as_empty():
    b, hq, hkv, d, cap = 3, 4, 1, 64, 150
    q, K, V = _inputs(b, hq, hkv, d, cap, 1, seed=30)
    lens = torch.tensor([[150], [151], [-5]], dtype=torch.int32, device="cuda")
    w = torch.zeros(b, hkv, cap, device="cuda")
    bk = _bk(b, hq, hkv, d, cap)
    try:
        bk.reserve_attend(weights=True, n_groups=1)
        o, lse = bk.attend(q, K, V, length=lens, weights=w)
        with pytest.raises(bkv.BkvError) as ei:
            bk.sync()
        assert ei.value.code == bkv.BKV_EINVAL
        (o64, l64, w64), (to, tl, tw) = reference(q, K, V, lens * torch.tensor([[1], [0], [0]], device="cuda"))
        check(o, o64, to, "o")
        check(lse, l64, tl, "lse")
        check(w, w64, tw, "weights")
        pl = torch.tensor([99], dtype=torch.int32, device="cuda")
        bk.attend_shared(q, K[:1, :, :98].contiguous(), V[:1, :, :98].contiguous(), K, V, prefix_len=pl,
                         length=torch.zeros_like(lens))
        with pytest.raises(bkv.BkvError) as ei:
            bk.sync()
        assert ei.value.code == bkv.BKV_EINVAL
    finally:
        bk.close()


def test_refusals():
    b, hq, hkv, d, cap = 4, 4, 2, 64, 100
    q, K, V = _inputs(b, hq, hkv, d, cap, 2, seed=31)
    lens = _lens(b, hkv, [100])
    o, w = torch.full_like(q, 3.0), torch.full((b, hkv, cap), 3.0, device="cuda")
    Kp, Vp = K[:2].contiguous(), V[:2].contiguous()
    pl = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    bk = _bk(b, hq, hkv, d, cap, window=8, n_beacons=0)

    def code_of(fn):
        with pytest.raises(bkv.BkvError) as ei:
            fn()
        return ei.value.code

    def attend(q_=q, n_q=2, K_=K, V_=V, scale=0.0):
        bkv.bkv_attend(bk.ctx, q_, n_q, K_, V_, lens, scale, o, None, w)

    def shared(n_groups=2, pcap=cap, plen=pl, Kp_=Kp):
        bkv.bkv_attend_shared(bk.ctx, q, 2, Kp_, Vp, plen, n_groups, pcap, K, V, lens, 0.0, o, None, w)

    odd = torch.empty(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:]
    try:
        assert code_of(attend) == bkv.BKV_ESTATE                      # no reservation yet
        bk.reserve_attend(n_q=2, n_groups=2, weights=True)
        assert code_of(lambda: attend(n_q=-1)) == bkv.BKV_EINVAL
        assert code_of(lambda: attend(q_=None)) == bkv.BKV_EINVAL
        assert code_of(lambda: attend(q_=odd)) == bkv.BKV_EINVAL
        for scale in (-1.0, math.nan, math.inf, 1e300, 1e-300):
            assert code_of(lambda: attend(scale=scale)) == bkv.BKV_EINVAL
        assert code_of(lambda: attend(n_q=1 << 27)) == bkv.BKV_EINVAL
        assert code_of(lambda: shared(n_groups=0)) == bkv.BKV_EINVAL
        assert code_of(lambda: shared(n_groups=3)) == bkv.BKV_EINVAL  # 3 does not divide the batch
        assert code_of(lambda: shared(pcap=0)) == bkv.BKV_EINVAL
        assert code_of(lambda: shared(plen=None)) == bkv.BKV_EINVAL
        assert code_of(lambda: shared(Kp_=None)) == bkv.BKV_EINVAL
        assert code_of(lambda: bk.reserve_attend(n_q=-1)) == bkv.BKV_EINVAL
        assert code_of(lambda: bk.reserve_attend(n_groups=3)) == bkv.BKV_EINVAL
        attend(n_q=0)                                                 # no queries: nothing to do
        # allocation failure: the workspace in place stays usable
        bkv.bkv_debug_fail_alloc(1)
        assert code_of(lambda: bk.reserve_attend(n_q=50, weights=True)) == bkv.BKV_ENOMEM
        bkv.bkv_debug_fail_alloc(0)
        # evict
        L = _lens(b, hkv, [100]).view(1, b, hkv)
        K5, V5, w5 = K[None], V[None], w[None]
        out = [torch.zeros_like(t) for t in (K5, V5, w5)]
        kept = torch.full((1, b, hkv, 50), -7, dtype=torch.int32, device="cuda")
        ev = lambda budget=50, Ko=out[0], Vo=out[1], wo=out[2], co=cap, K_=K5: bkv.bkv_evict(  # noqa: E731
            bk.ctx, K_, V5, w5, L, budget, Ko, Vo, wo, co, kept)
        assert code_of(lambda: ev(budget=7)) == bkv.BKV_EINVAL        # below the window
        assert code_of(lambda: ev(co=49)) == bkv.BKV_EINVAL           # no room for the kept rows
        assert code_of(lambda: ev(K_=None)) == bkv.BKV_EINVAL
        assert code_of(lambda: ev(Ko=K5)) == bkv.BKV_EINVAL           # one output in place, the others not
        assert code_of(lambda: ev(Vo=out[0])) == bkv.BKV_EINVAL       # two outputs in one buffer
        assert code_of(lambda: ev(Ko=K5, Vo=V5, wo=w5, co=cap - 1)) == bkv.BKV_EINVAL
        with pytest.raises(ValueError):
            bk.evict(K5, V5, w5, L=L, budget=50, K_out=out[0])
        with pytest.raises(ValueError):
            bk.attend(q[:, :2], K, V, length=lens)
        with pytest.raises(ValueError):
            bk.attend(q, K[:, :, :-1].contiguous(), V, length=lens)
        with pytest.raises(ValueError):
            bk.attend(q, K.transpose(0, 1), V, length=lens)           # not contiguous
        with pytest.raises(TypeError):
            bk.attend(q.float(), K, V, length=lens)
        with pytest.raises(TypeError):
            bk.attend(q.cpu(), K, V, length=lens)
        bk.sync()
        assert bool((o == 3).all()) and bool((w == 3).all()) and bool((kept == -7).all())
        assert not any(bool(t.any()) for t in out)
        bk.attend(q, K, V, length=lens, weights=w)
        bk.sync()
    finally:
        bkv.bkv_debug_fail_alloc(0)
        bk.close()


@pytest.mark.parametrize("groups", [0, 2])
@pytest.mark.parametrize("most", [300, 70, 40])
def test_a_reservation_serves_every_smaller_call(groups, most):
    """Fewer queries can need more room (their logits are kept); the reservation covers them all."""
    b, hq, hkv, d, cap = 4, 8, 2, 64, 12000
    lens = _lens(b, hkv, [700, 333, 0, 12000])
    plens = torch.tensor([150, 0], dtype=torch.int32, device="cuda")
    bk = _bk(b, hq, hkv, d, cap)
    try:
        bk.reserve_attend(n_q=most, n_groups=groups, weights=True)
        for n_q in (1, 2, 4, 7, 8, 9, 16, 17, 31, 32, 33, 39, 40, 63, 64, 65, 70, 100, 128, 129, 255, 256, 257, 299, 300):
            if n_q > most:
                continue
            q, K, V = _inputs(b, hq, hkv, d, cap, n_q, seed=50)
            w = torch.zeros(b, hkv, cap, device="cuda")
            if groups:
                Kp, Vp = _inputs(groups, hq, hkv, d, 150, 1, seed=51)[1:]
                bk.attend_shared(q, Kp, Vp, K, V, prefix_len=plens, length=lens, weights=w)
            else:
                bk.attend(q, K, V, length=lens, weights=w)
                # every query that sees a row spreads a weight of 1
                rows = torch.clamp(lens, max=n_q).float() * (hq // hkv)
                bk.sync()
                torch.testing.assert_close(w.sum(-1), rows, rtol=2.0 ** -11, atol=1e-6)
        bk.sync()
    finally:
        bk.close()


def test_more_tiles_than_fit_31_bits_are_refused():
    """A prefix as long as the limits allow times as many row blocks: refused before anything is read."""
    b, cap, n_q = 64, 16, 1 << 20
    bk = _bk(b, 1, 1, 64, cap)
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda")  # the addresses only have to be valid
    n = torch.zeros(b, dtype=torch.int32, device="cuda")
    try:
        with pytest.raises(bkv.BkvError) as ei:
            bkv.bkv_attend_shared(bk.ctx, x, n_q, x, x, n, 1, 1 << 29, x, x, n, 0.0, x)
        assert ei.value.code == bkv.BKV_EINVAL
        with pytest.raises(bkv.BkvError) as ei:  # one prefix of 2^30 rows is past the row limit
            bkv.bkv_attend_shared(bk.ctx, x, 1, x, x, n, 1, 1 << 30, x, x, n, 0.0, x)
        assert ei.value.code == bkv.BKV_EINVAL
        bk.sync()
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
def test_output_aligned_to_16_bytes_only(d):
    b, hq, hkv, cap, n_q = 2, 8, 2, 500, 100
    lens = _lens(b, hkv, [500, 333, 100, 90])
    q, K, V = _inputs(b, hq, hkv, d, cap, n_q, seed=60)
    _poison(K, V, lens)
    bk = _bk(b, hq, hkv, d, cap)
    try:
        o, _, _ = run_and_check(bk, q, K, V, lens)
        room = torch.full((q.numel() + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[8:-8].view(q.shape)
        assert out.data_ptr() % 32 == 16
        bk.attend(q, K, V, length=lens, o_out=out)
        bk.sync()
        assert torch.equal(out, o) and bool((room[:8] == 7).all()) and bool((room[-8:] == 7).all())
    finally:
        bk.close()


@pytest.mark.parametrize("kind", ["random", "equal", "rising", "falling"])
@pytest.mark.parametrize("cap", [10241, 16384, 20480, 20481, 27000, 32768])
def test_evict_long_instances(cap, kind):
    """Instances whose rows several blocks share: lengths that leave blocks without rows or with one, ties that
    run across blocks."""
    g = torch.Generator(device="cuda").manual_seed(cap)
    budget = 700
    shape = (1, 2, 6)
    K, V = (torch.randn(*shape, cap, 64, generator=g, device="cuda").bfloat16() for _ in "KV")
    if kind == "random":
        w = torch.exp(2 * torch.randn(*shape, cap, generator=g, device="cuda"))
    elif kind == "equal":
        w = torch.full((*shape, cap), 0.25, device="cuda")
        w[..., ::7] = 0.5
    else:
        w = torch.arange(cap, device="cuda").float().expand(*shape, cap).contiguous()
        w = w if kind == "rising" else -w
    L = torch.tensor([cap, cap - 1, 0, 1, 700, 701, 1025, 2049, 4097, cap // 2 + 1, 8193, 10000], dtype=torch.int32,
                     device="cuda").view(shape)
    bk = _bk(2, 12, 6, 64, cap, window=16, n_beacons=0, n_prefix=4)
    try:
        _check_evict(bk, K, V, w, L, budget)
        bad = L.clone()
        bad[0, 0, 0], bad[0, 1, 5] = cap + 1, -3
        out = [torch.zeros(*shape, budget, 64, dtype=torch.bfloat16, device="cuda") for _ in "KV"]
        kept, new = bk.evict(K, V, w, L=bad, budget=budget, K_out=out[0], V_out=out[1],
                             weights_out=torch.zeros(*shape, budget, device="cuda"))
        with pytest.raises(bkv.BkvError):
            bk.sync()
        for e in (0, 11):
            assert int(new.flatten()[e]) == 0 and bool((kept.view(12, -1)[e] == -1).all())
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_inst", [152, 153, 304, 306, 608, 610, 1300])
def test_evict_in_place_of_many_instances(n_inst, d):
    """From more instances on, each has fewer threads."""
    g = torch.Generator(device="cuda").manual_seed(n_inst)
    cap, budget, hkv = 90, 61, 1 if n_inst % 2 else 2
    shape = (1, n_inst // hkv, hkv)
    K, V = (torch.randn(*shape, cap, d, generator=g, device="cuda").bfloat16() for _ in "KV")
    w = torch.rand(*shape, cap, generator=g, device="cuda")
    L = torch.randint(0, cap + 1, shape, generator=g, device="cuda", dtype=torch.int32)
    bk = _bk(shape[1], hkv, hkv, d, cap, window=4, n_beacons=0, n_prefix=2)
    try:
        _check_evict(bk, K, V, w, L, budget)
    finally:
        bk.close()
