"""Caches held in 4 bits: bkv_pack4, bkv_unpack4, bkv_attend4 and bkv_evict4 against plain implementations in 64 bits.

bkv_pack4 is exact: each of its three roundings is the rounding of the exact value, so codes and scales have to be
equal bit for bit.  bkv_unpack4 rounds an exact sum once, in fp32 (2^-24) and then to bf16: equal to the bf16 rounding
of the 64-bit value but where that lies within 2^-24 of a tie, so off by at most one bf16 step there.

bkv_attend4 on the codes, with B_j = scale * sum_g (step_jg sum n |q| + |low_jg| sum |q|), the size of a logit's terms:
- a logit takes at most 32 additions of a group's exact products, 8 of its groups and the queries' sum of 8 + 2, each
  off by at most 2^-23 of the terms so far: 2^-16 B covers them;
- lse and weights: as for bkv_attend (tests/test_gpu_attend.py) with B for S; delta = 2 * 2^-16 B + 2^-14;
- o: p and its products with the steps are rounded to fp16 (2^-11 each), the result to bf16 (2^-8).  p stands as p 2^E,
  2^E being 2^8 / max step at least, or 2^11, and the sum of p being 1 at least: a rounding below fp16's normal range is
  off by 2^-25-E, of a product times 15, of p times a step and 15 or times a low:
  |o - o64| <= 2^-8 |o| + sum_j p_j ((2^-10 + 2 delta) step_j n_j + (2^-11 + 2 delta) |low_j|)
               + 2^-25-E sum_j (15 (1 + step_j) + |low_j|).
More rows read the values as fp16 numbers, with S_j = scale sum |q k_j|:
- a logit takes twice the head_dim additions (K is a sum of two terms, off by 2^-22 of itself): 2^-15 S, and query
  elements below 2^-14 are off by 2^-25 at most: scale sum |k| 2^-25;
- o: the weights (2^-11; below 2^-14 of the first key's by 2^-25 of it) and V (2^-11; below 2^-14 by 2^-25) are rounded:
  |o - o64| <= 2^-8 |o| + (2^-10 + 2 delta) sum p |v| + 2^-25 (len max |v| + 1).
"""
import math

import pytest
import torch

from paper_2609_04971_gb300 import bkv
from tests import test_gpu_attend as ga

pytestmark = pytest.mark.gpu

DEV = "cuda"


# ------------------------------------------------------------------------------------------ the format, by itself
def half64(x):
    """Nearest fp16 numbers of fp64 x, ties to even, limited to 65504."""
    a = x.abs().clamp(max=65504.0)
    e = (a.view(torch.int64) >> 52).clamp(min=1023 - 14)      # biased exponent, of the smallest normal number below
    unit = ((e - 10) << 52).view(torch.float64)
    return torch.copysign((torch.round(a / unit) * unit).clamp(max=65504.0), x)


def pack64(x):
    """codes [.., d], step and low [.., d / 32] of bf16 rows, in 64 bits."""
    g = x.double().clamp(-65504.0, 65504.0).unflatten(-1, (-1, 32))
    low = half64(x.double().unflatten(-1, (-1, 32)).amin(-1))
    step = half64((x.double().unflatten(-1, (-1, 32)).amax(-1) - low).clamp(min=0) / 15)
    n = torch.round((x.double().unflatten(-1, (-1, 32)) - low[..., None]) / step.clamp(min=2.0 ** -40)[..., None])
    n = torch.where(step[..., None] > 0, n, torch.zeros_like(g)).clamp(0, 15)
    return n.flatten(-2), step, low


def order(d, which):
    """Element of code x of word w, [d / 8][8]."""
    w, x = torch.arange(d // 8, device=DEV)[:, None], torch.arange(8, device=DEV)[None]
    if which == 0:
        return 32 * (w % (d // 32)) + 8 * (w // (d // 32)) + x
    return w + x * (d // 8)


def to_words(code, which):
    d = code.shape[-1]
    c = code.long()[..., order(d, which)]  # [.., d / 8, 8]
    byte = c[..., 0::2] + 16 * c[..., 1::2]
    return byte.flatten(-2).to(torch.uint8)


def from_words(words, which):
    d = 2 * words.shape[-1]
    b = words.long().unflatten(-1, (d // 8, 4))
    c = torch.stack((b % 16, b // 16), -1).flatten(-2)
    out = torch.empty(*words.shape[:-1], d, dtype=torch.long, device=words.device)
    out[..., order(d, which).flatten()] = c.flatten(-2)
    return out


def values64(words, S4, which):
    """(values, step * code, low) of rows, [.., d] each, in 64 bits."""
    sc = S4[..., which, :, :].double().repeat_interleave(32, -2)
    sn = sc[..., 0] * from_words(words, which)
    return sc[..., 1] + sn, sn, sc[..., 1]


def new_cache(*lead, d, fill=0):
    K4, V4 = (torch.full((*lead, d // 2), fill, dtype=torch.uint8, device=DEV) for _ in "KV")
    return K4, V4, torch.zeros(*lead, 2, d // 32, 2, dtype=torch.float16, device=DEV)


def packed(K, V):
    """4-bit caches of bf16 ones, by the 64-bit rules."""
    K4, V4, S4 = new_cache(*K.shape[:-1], d=K.shape[-1])
    for which, (x, w) in enumerate(((K, K4), (V, V4))):
        n, step, low = pack64(x)
        w.copy_(to_words(n, which))
        S4[..., which, :, 0], S4[..., which, :, 1] = step, low
    return K4, V4, S4


def rows(*shape, seed=0, spread=0.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(*shape, generator=g, device=DEV)
    if spread:
        x = x * torch.exp(spread * torch.randn(*shape[:-1], 1, generator=g, device=DEV))
    return x.bfloat16()


# ------------------------------------------------------------------------------------------ pack and unpack
def check_pack(bk, K, V, first, lens, cap):
    b, hkv, n, d = K.shape
    K4, V4, S4 = new_cache(b, hkv, cap, d=d, fill=0xA5)
    S4.fill_(3.0)
    want = [t.clone() for t in (K4, V4, S4)]
    bk.pack4(K, V, K4, V4, S4, first=first, length=lens)
    K2, V2 = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    want2 = [K2.clone(), V2.clone()]
    bk.unpack4(K4, V4, S4, K2, V2, first=first, length=lens)
    bk.sync()
    for x in range(b):
        for y in range(hkv):
            f = 0 if first is None else int(first[x, y])
            m = max(0, min(n, int(lens[x, y]) - f))
            for which, src in enumerate((K, V)):
                code, step, low = pack64(src[x, y, :m])
                want[which][x, y, f:f + m] = to_words(code, which)
                want[2][x, y, f:f + m, which, :, 0], want[2][x, y, f:f + m, which, :, 1] = step, low
                v = low.repeat_interleave(32, -1) + step.repeat_interleave(32, -1) * code
                want2[which][x, y, :m] = v.bfloat16()
    for got, w, what in zip((K4, V4, S4), want, ("K4", "V4", "S4")):
        assert torch.equal(got, w), f"{what}: {int((got != w).sum())} of {got.numel()} differ"
    for got, w in zip((K2, V2), want2):
        off = (got.double() - w.double()).abs()
        assert float((off > 0).double().mean()) < 1e-3 and bool((off <= 2.0 ** -7 * w.double().abs()).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,cap", [(1, 5), (7, 40), (33, 33), (130, 200)])
def test_pack_and_unpack(d, n, cap):
    """Every mix of rows that fit, rows past the length, and caches that take nothing."""
    b, hkv = 3, 3
    K, V = rows(b, hkv, n, d, seed=n, spread=2.0), rows(b, hkv, n, d, seed=n + 1, spread=2.0)
    K[0, 0, 0] = 0.0
    V[0, 1, 0, :32] = 0.3          # a constant group
    V[1, 1, 0] = torch.arange(d, device=DEV) % 16 * 0.25 + 1  # exact codes
    lens = ga._lens(b, hkv, [cap, 0, n, min(cap, n + 1), 1, cap, n // 2, cap - 1, cap])
    first = (lens - torch.tensor([0, 0, n, 1, 0, 2, n // 3, n, n // 2], device=DEV).view(b, hkv)).clamp(min=0).int()
    bk = ga._bk(b, hkv, hkv, d, cap)
    try:
        check_pack(bk, K, V, first, lens, cap)
        check_pack(bk, K, V, None, lens, cap)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
def test_pack_ties_and_extremes(d):
    """Codes on and next to their borders, the largest and smallest numbers, signs of zero."""
    b, hkv, n = 1, 2, 3000
    g = torch.Generator(device=DEV).manual_seed(3)
    K = torch.randint(-40, 41, (b, hkv, n, d), generator=g, device=DEV).float()  # multiples: many exact ties
    K *= torch.pow(2.0, torch.randint(-12, 9, (b, hkv, n, 1), generator=g, device=DEV).float())
    V = torch.randint(-7, 8, (b, hkv, n, d), generator=g, device=DEV).float()
    V[:, :, :500] *= torch.pow(2.0, -torch.randint(0, 40, (b, hkv, 500, d), generator=g, device=DEV).float())
    V[:, :, 500:600] *= 2.0 ** 100
    V[:, :, 600:700] *= 2.0 ** -120
    V[:, :, 700] = -0.0
    V[:, :, 701] = 3e38
    V[:, :, 702] = -3e38
    V[:, :, 703, ::2] = 65504
    lens = ga._lens(b, hkv, [n])
    bk = ga._bk(b, hkv, hkv, d, n)
    try:
        check_pack(bk, K.bfloat16(), V.bfloat16(), None, lens, n)
    finally:
        bk.close()


def test_pack_lengths_out_of_range():
    b, hkv, d, cap, n = 2, 2, 64, 20, 4
    K, V = rows(b, hkv, n, d), rows(b, hkv, n, d, seed=1)
    bk = ga._bk(b, hkv, hkv, d, cap)
    try:
        for first, lens in (([0, 0, 0, 0], [4, 21, 4, 4]), ([0, 0, 0, 0], [4, -1, 4, 4]), ([0, -1, 0, 0], [4, 4, 4, 4]),
                            ([0, 5, 0, 0], [4, 4, 4, 4])):
            f, L = (torch.tensor(v, dtype=torch.int32, device=DEV).view(b, hkv) for v in (first, lens))
            K4, V4, S4 = new_cache(b, hkv, cap, d=d, fill=1)
            bk.pack4(K, V, K4, V4, S4, first=f, length=L)
            with pytest.raises(bkv.BkvError) as ei:
                bk.sync()
            assert ei.value.code == bkv.BKV_EINVAL
            assert bool((K4[0, 1] == 1).all()) and bool((S4[0, 1] == 0).all())
            assert torch.equal(K4[1, 1, :4], to_words(pack64(K[1, 1])[0], 0))
            out = torch.full_like(K, 2.0)
            bk.unpack4(K4, V4, S4, out, torch.full_like(V, 2.0), first=f, length=L)
            with pytest.raises(bkv.BkvError):
                bk.sync()
            assert bool((out[0, 1] == 2).all())
        bk.pack4(K[:, :, :0], V[:, :, :0], K4, V4, S4, length=L)  # no rows
        bk.sync()
    finally:
        bk.close()


# ------------------------------------------------------------------------------------------ attention
def reference4(q, K4, V4, S4, lens, scale=None, many=False):
    b, hq, n_q, d = q.shape
    hkv, cap = K4.shape[1:3]
    G = hq // hkv
    scale = scale or 1 / math.sqrt(d)
    o = torch.zeros(b, hq, n_q, d, dtype=torch.float64, device=DEV)
    lse = torch.full((b, hq, n_q), -math.inf, dtype=torch.float64, device=DEV)
    w = torch.zeros(b, hkv, cap, dtype=torch.float64, device=DEV)
    to, tl, tw = torch.zeros_like(o), torch.zeros_like(lse), torch.zeros_like(w)
    for x in range(b):
        for y in range(hkv):
            n = int(lens[x, y])
            if n == 0:
                continue
            k, k_sn, k_low = values64(K4[x, y, :n], S4[x, y, :n], 0)
            v, v_sn, v_low = values64(V4[x, y, :n], S4[x, y, :n], 1)
            i = torch.arange(n_q, device=DEV).repeat(G)[:, None]
            seen = torch.arange(n, device=DEV)[None] < n - n_q + 1 + i
            qq = q[x, y * G:(y + 1) * G].reshape(G * n_q, d).double()
            z = (qq @ k.T * scale).masked_fill(~seen, -math.inf)
            terms = k.abs() if many else k_sn + k_low.abs()
            err = qq.abs() @ terms.T * scale * 2.0 ** (-15 if many else -16)
            if many:
                err = err + k.abs().sum(-1) * scale * 2.0 ** -25
            err = err.masked_fill(~seen, 0).amax(-1)
            t = torch.logsumexp(z, -1)
            p = torch.exp(z - torch.where(t == -math.inf, 0.0, t)[:, None])
            delta = (2 * err + 2.0 ** -14)[:, None]
            r = slice(y * G, (y + 1) * G)
            oo = p @ v
            o[x, r] = oo.view(G, n_q, d)
            if many:
                off = (2.0 ** -10 + 2 * delta) * (p @ v.abs()) + 2.0 ** -25 * (n * v.abs().max() + 1)
            else:
                step = S4[x, y, :n, 1, :, 0].double()
                unit = 2.0 ** -25 * max(float(step.max()) * 2.0 ** -8, 2.0 ** -11)  # 2^-25-E
                off = ((2.0 ** -10 + 2 * delta) * (p @ v_sn) + (2.0 ** -11 + 2 * delta) * (p @ v_low.abs())
                       + unit * float((15 * (1 + step) + S4[x, y, :n, 1, :, 1].double().abs()).amax(-1).sum()))
            to[x, r] = (2.0 ** -8 * oo.abs() + off).view(G, n_q, d)
            lse[x, r] = t.view(G, n_q)
            tl[x, r] = (err + 2.0 ** -15 + 2.0 ** -22 * t.abs()).view(G, n_q)
            w[x, y, :n] = p.sum(0)
            tw[x, y, :n] = (p * delta).sum(0) + (G * n_q + 8) * 2.0 ** -24 * w[x, y, :n]
    return (o, lse, w), (to, tl, tw)


def run4(bk, q, cache, lens, *, weights=True, scale=None, ref=None):
    K4, V4, S4 = cache
    w0 = torch.rand(*K4.shape[:3], device=DEV) + 0.25  # a weight below fp32's range added to 0 would be lost
    w = w0.clone() if weights else None
    bk.reserve_attend4(n_q=q.shape[2], weights=weights)
    o, lse = bk.attend4(q, K4, V4, S4, length=lens, weights=w, scale=scale)
    bk.sync()
    (o64, l64, w64), (to, tl, tw) = ref or reference4(q, K4, V4, S4, lens, scale)
    ga.check(lse, l64, tl, "lse")
    ga.check(o, o64, to, "o")
    if weights:
        past = torch.arange(K4.shape[2], device=DEV) >= lens[..., None]
        assert torch.equal(w[past], w0[past]), "weights past the length were touched"
        ga.check(w, w0.double() + w64, tw + 2.0 ** -23 * (w0 + w64), "weights")
    return o, lse, w


def poison(cache, lens):
    K4, V4, S4 = cache
    for x in range(K4.shape[0]):
        for y in range(K4.shape[1]):
            n = int(lens[x, y])
            K4[x, y, n:], V4[x, y, n:] = 0xFF, 0xFF
            S4[x, y, n:] = math.nan
            S4[x, y, n::2] = math.inf


def case(b, hq, hkv, d, cap, n_q, lens, seed=0, spread=0.5, std=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (std * torch.randn(b, hq, n_q, d, generator=g, device=DEV)).bfloat16()
    K, V = (rows(b, hkv, cap, d, seed=seed + i, spread=spread) for i in (1, 2))
    cache = packed(K, V)
    poison(cache, lens)
    return q, cache


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 9, 16, 17])
def test_single_tokens(d, G):
    b, hkv, cap = 4, 2, 700
    lens = ga._lens(b, hkv, [1, 15, 16, 17, 700, 0, 129, 300])
    q, cache = case(b, G * hkv, hkv, d, cap, 1, lens, seed=G)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        run4(bk, q, cache, lens)
        run4(bk, q, cache, lens, weights=False, scale=0.03)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(1, 7), (4, 2), (4, 8), (5, 5), (3, 11), (2, 40), (8, 10)])
def test_several_tokens(d, G, n_q):
    """Causal among the new tokens, one or several row blocks, caches shorter than the new tokens."""
    b, hkv, cap = 3, 2, 400
    lens = ga._lens(b, hkv, [400, n_q - 1, n_q, 2, 131, 256])
    q, cache = case(b, G * hkv, hkv, d, cap, n_q, lens, seed=n_q)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        run4(bk, q, cache, lens, weights=G * n_q <= 48)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,weights", [(4, 13, True), (4, 25, False), (1, 97, True), (8, 40, True), (2, 300, False),
                                           (5, 130, True)])
def test_many_rows_are_read_as_fp16(d, G, n_q, weights):
    b, hkv, cap = 2, 2, 750
    lens = ga._lens(b, hkv, [750, 301, 129, 5])
    q, cache = case(b, G * hkv, hkv, d, cap, n_q, lens, seed=n_q)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        run4(bk, q, cache, lens, weights=weights, ref=reference4(q, *cache, lens, many=True))
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
def test_references_move_with_many_rows(d):
    """Logits that rise by hundreds along a cache, in fp16: the references follow before a weight is too large."""
    b, hq, hkv, cap, n_q = 2, 4, 2, 900, 150
    lens = ga._lens(b, hkv, [900, 513, 899, 640])
    g = torch.Generator(device=DEV).manual_seed(9)
    ramp = torch.linspace(0.1, 12, cap, device=DEV)[:, None]
    u = torch.randn(b, hkv, 1, d, generator=g, device=DEV)
    K = (u * ramp + torch.randn(b, hkv, cap, d, generator=g, device=DEV)).bfloat16()
    V = torch.randn(b, hkv, cap, d, generator=g, device=DEV).bfloat16()
    q = (torch.randn(b, hq, n_q, d, generator=g, device=DEV) + 4 * u.repeat_interleave(2, 1)).bfloat16()
    cache = packed(K, V)
    poison(cache, lens)
    bk = ga._bk(b, hq, hkv, d, cap)
    try:
        for qq in (q, -q):
            run4(bk, qq, cache, lens, ref=reference4(qq, *cache, lens, many=True))
    finally:
        bk.close()


@pytest.mark.parametrize("d,G,n_q", [(128, 4, 1), (64, 7, 1), (128, 8, 2)])
def test_long_caches_in_parts(d, G, n_q):
    """Caches that many blocks share: parts of different lengths, one of them short."""
    b, hkv, cap = 1, 2, 20011
    lens = ga._lens(b, hkv, [20011, 77])
    q, cache = case(b, G * hkv, hkv, d, cap, n_q, lens, seed=5)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        first = run4(bk, q, cache, lens, weights=True)
        w = torch.zeros(b, hkv, cap, device=DEV)
        again = bk.attend4(q, *cache, length=lens, weights=w)
        bk.sync()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
def test_references_and_step_scales_move(d):
    """Logits that rise by hundreds along a cache, steps of V that span 2^24, weights concentrated on tiny values."""
    b, hq, hkv, cap = 2, 8, 2, 900
    lens = ga._lens(b, hkv, [900, 513, 899, 640])
    g = torch.Generator(device=DEV).manual_seed(9)
    ramp = torch.linspace(0.1, 12, cap, device=DEV)[:, None]
    K = (torch.randn(b, hkv, 1, d, generator=g, device=DEV) * ramp
         + torch.randn(b, hkv, cap, d, generator=g, device=DEV)).bfloat16()
    V = torch.randn(b, hkv, cap, d, generator=g, device=DEV)
    V *= torch.pow(2.0, torch.randint(-12, 12, (b, hkv, cap, 1), generator=g, device=DEV).float())
    V[:, :, -200:] *= 2.0 ** -12
    q = (torch.randn(b, hkv, 1, d, generator=g, device=DEV).repeat_interleave(4, 1).repeat(1, 1, 1, 1)
         + K[:, :, :1].repeat_interleave(4, 1) * 20).bfloat16()
    cache = packed(K, V.bfloat16())
    poison(cache, lens)
    bk = ga._bk(b, hq, hkv, d, cap)
    try:
        run4(bk, q, cache, lens)
        run4(bk, -q, cache, lens)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,level", [(4, 1, -1), (4, 1, 1), (5, 3, -1), (2, 60, -1)])
def test_logits_far_from_zero(d, G, n_q, level):
    """All logits hundreds below (or above) 0, in caches so short that most of a block's warps have no keys."""
    b, hkv, cap = 2, 2, 333
    lens = ga._lens(b, hkv, [1, 40, 333, 129])
    g = torch.Generator(device=DEV).manual_seed(4)
    u = torch.randn(b, hkv, 1, d, generator=g, device=DEV)
    K = (4 * u + torch.randn(b, hkv, cap, d, generator=g, device=DEV)).bfloat16()
    q = (level * 8 * u.repeat_interleave(G, 1) + torch.randn(b, G * hkv, n_q, d, generator=g, device=DEV)).bfloat16()
    cache = packed(K, rows(b, hkv, cap, d, seed=5))
    poison(cache, lens)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        many = G * n_q > 96
        run4(bk, q, cache, lens, weights=not many, ref=reference4(q, *cache, lens, many=many))
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
def test_extreme_queries_and_constant_rows(d):
    """Queries of every magnitude (with a scale to match), zero queries, rows of one value, all-zero caches."""
    b, hq, hkv, cap = 4, 8, 2, 150
    lens = ga._lens(b, hkv, [150, 31])
    q, cache = case(b, hq, hkv, d, cap, 1, lens, seed=2, spread=0.0)
    q[1] = (q[1].double() * 2.0 ** 60).bfloat16()
    q[2] = (q[2].double() * 2.0 ** -60).bfloat16()
    q[3] = 0
    q[0, 0, 0, 1:] *= 2.0 ** -20  # one element far above the others
    bk = ga._bk(b, hq, hkv, d, cap)
    try:
        run4(bk, q, cache, lens, scale=2.0 ** -62)
        q[1] = 0
        run4(bk, q, cache, lens)
        K, V = (torch.full((b, hkv, cap, d), x, device=DEV).bfloat16() for x in (0.7, 0.0))
        V[:, :, 100:] = -3.1
        run4(bk, q, packed(K, V), lens)
    finally:
        bk.close()


def test_lengths_out_of_range_count_as_empty():
    b, hq, hkv, d, cap = 2, 4, 2, 64, 100
    lens = torch.tensor([[100, 101], [-1, 50]], dtype=torch.int32, device=DEV)
    ok = torch.tensor([[100, 0], [0, 50]], dtype=torch.int32, device=DEV)
    q, cache = case(b, hq, hkv, d, cap, 1, ok)
    bk = ga._bk(b, hq, hkv, d, cap)
    try:
        for n_q in (1, 60):
            qq = q.expand(-1, -1, n_q, -1).contiguous()
            bk.reserve_attend4(n_q=n_q)
            o, lse = bk.attend4(qq, *cache, length=lens)
            with pytest.raises(bkv.BkvError) as ei:
                bk.sync()
            assert ei.value.code == bkv.BKV_EINVAL
            want, want_l = bk.attend4(qq, *cache, length=ok)
            bk.sync()
            assert torch.equal(o, want) and torch.equal(lse, want_l) and bool((o[0, 2:] == 0).all())
    finally:
        bk.close()


def test_refusals():
    b, hq, hkv, d, cap = 2, 4, 2, 64, 96
    lens = ga._lens(b, hkv, [96])
    q, (K4, V4, S4) = case(b, hq, hkv, d, cap, 1, lens)
    o, lse, w = torch.zeros_like(q), torch.zeros(b, hq, 1, device=DEV), torch.zeros(b, hkv, cap, device=DEV)
    bk = ga._bk(b, hq, hkv, d, cap)

    def refused(code, f, *a):
        with pytest.raises(bkv.BkvError) as ei:
            f(bk.ctx, *a)
        assert ei.value.code == code, str(ei.value)

    try:
        refused(bkv.BKV_ESTATE, bkv.bkv_attend4, q, 1, K4, V4, S4, lens, 0.0, o, lse, w)
        bk.reserve_attend4(n_q=1, weights=True)
        bad = bkv.BKV_EINVAL
        for a in ((None, 1, K4, V4, S4, lens, 0.0, o), (q, 1, K4, None, S4, lens, 0.0, o),
                  (q, 1, K4, V4, None, lens, 0.0, o), (q, 1, K4, V4, S4, None, 0.0, o),
                  (q, 1, K4, V4, S4, lens, 0.0, None), (q, -1, K4, V4, S4, lens, 0.0, o),
                  (q, 1, K4, V4, S4, lens, -1.0, o), (q, 1, K4, V4, S4, lens, math.nan, o),
                  (q, 1, K4, V4, S4, lens, 1e39, o), (q, 1 << 27, K4, V4, S4, lens, 0.0, o),
                  (q, 1, K4.view(-1)[8:], V4, S4, lens, 0.0, o), (q, 1, K4, V4, S4, lens, 0.0, q),
                  (q, 1, K4, V4, S4, lens, 0.0, K4.view(torch.bfloat16)),
                  (q, 1, K4, V4, S4, lens, 0.0, o, S4.view(torch.float32)),
                  (q, 1, K4, V4, S4, lens, 0.0, o, lse, V4.view(torch.float32)),
                  (q, 1, K4, V4, S4, lens, 0.0, o, lse, lens.view(torch.float32))):
            refused(bad, bkv.bkv_attend4, *a)
        K, V = rows(b, hkv, 3, d), rows(b, hkv, 3, d)
        for a in ((None, V, 3, None, lens, K4, V4, S4), (K, V, 3, None, None, K4, V4, S4),
                  (K, V, -1, None, lens, K4, V4, S4), (K, V, 1 << 30, None, lens, K4, V4, S4),
                  (K, V, 3, None, lens, K4, K4, S4), (K, V, 3, None, lens, K.view(torch.uint8), V4, S4),
                  (K, V, 3, lens, lens, K4, lens.view(torch.uint8), S4),
                  (K, V, 3, None, lens, K4, V4.view(-1)[4:], S4)):
            refused(bad, bkv.bkv_pack4, *a)
        for a in ((K4, V4, S4, 3, None, lens, K, K), (K4, V4, S4, 3, None, lens, K4.view(torch.bfloat16), V),
                  (K4, V4, S4, 3, None, lens, K, None), (K4, None, S4, 3, None, lens, K, V)):
            refused(bad, bkv.bkv_unpack4, *a)
        kept = torch.zeros(b, hkv, 50, dtype=torch.int32, device=DEV)
        for a in ((K4, V4, None, w, lens, 50, K4, V4, S4, w, cap, kept),
                  (K4, V4, S4, w, lens, 50, K4, V4, S4, w, 60, kept),
                  (K4, V4, S4, w, lens, 0, K4, V4, S4, w, cap, kept),
                  (K4, K4, S4, w, lens, 50, K4, K4, S4, w, cap, kept),
                  (K4, V4, S4, w, lens, 50, K4, V4, S4.clone(), w, cap, kept)):
            refused(bad, bkv.bkv_evict4, *a)
        with pytest.raises(ValueError):
            bk.attend4(q, K4[:, :, :-1], V4, S4, length=lens)
        with pytest.raises(TypeError):
            bk.attend4(q, K4.view(torch.int8), V4, S4, length=lens)
        with pytest.raises(ValueError):
            bk.pack4(K[:, :1], V, K4, V4, S4, length=lens)
        with pytest.raises(ValueError):
            bk.evict4(K4, V4, S4, w, L=lens, budget=50, K4_out=K4)
        bk.sync()
        bk.attend4(q[:, :, :0], K4, V4, S4, length=lens)  # no queries
        bk.sync()
    finally:
        bk.close()


# ------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n_layers,b,hkv,cap,budget", [(1, 1, 1, 300, 64), (2, 3, 2, 1100, 900), (4, 10, 4, 200, 37),
                                                       (8, 10, 8, 70, 64)])
def test_eviction_moves_what_the_bf16_eviction_keeps(d, in_place, n_layers, b, hkv, cap, budget):
    """The rows kept, the weights and the lengths are those of bkv_evict; codes and scales move bit for bit."""
    shape, window, n_prefix = (n_layers, b, hkv), 8, 3
    g = torch.Generator(device=DEV).manual_seed(cap)
    K4, V4 = (torch.randint(0, 256, (*shape, cap, d // 2), generator=g, dtype=torch.uint8, device=DEV) for _ in "KV")
    S4 = torch.randn(*shape, cap, 2, d // 32, 2, generator=g, device=DEV).half()
    w = torch.rand(*shape, cap, generator=g, device=DEV)
    L = torch.randint(0, cap + 1, shape, generator=g, device=DEV).int()
    L.view(-1)[0] = cap
    cap_out = cap if in_place else budget + 5
    bk = ga._bk(b, hkv, hkv, d, cap, n_layers=n_layers, n_beacons=0, window=window, n_prefix=n_prefix)
    bf = torch.zeros(*shape, cap, d, device=DEV).bfloat16()
    bf2, w2 = bf.clone(), w.clone()
    want_kept, want_len = bk.evict(bf, bf2, w2, L=L, budget=budget)
    src = [t.clone() for t in (K4, V4, S4)]
    try:
        if in_place:
            out, wo = (K4, V4, S4), w
            kept, length = bk.evict4(K4, V4, S4, w, L=L, budget=budget)
        else:
            out = [torch.full((*shape, cap_out, *t.shape[4:]), 1, dtype=t.dtype, device=DEV) for t in src]
            wo = torch.full((*shape, cap_out), 9.0, device=DEV)
            kept, length = bk.evict4(K4, V4, S4, w, L=L, budget=budget, K4_out=out[0], V4_out=out[1], S4_out=out[2],
                                     weights_out=wo)
        bk.sync()
        assert torch.equal(kept, want_kept) and torch.equal(length, want_len)
        n = min(cap, cap_out)
        assert torch.equal(wo[..., :n], w2[..., :n])
        for s, t in zip(src, out):
            s, t = s.flatten(0, 2).flatten(2), t.flatten(0, 2).flatten(2)
            for e in range(s.shape[0]):
                rows_ = kept.flatten(0, 2)[e]
                rows_ = rows_[rows_ >= 0].long()
                assert torch.equal(t[e, :rows_.numel()], s[e, rows_])
                if not in_place:
                    assert bool((t[e, rows_.numel():] == 1).all())
    finally:
        bk.close()


# ------------------------------------------------------------------------------------------ together
def test_a_decode_loop_over_4_bit_caches():
    """Prompt rows packed, tokens appended one by one, attention with weights, an eviction, and on: the attention always
    agrees with the 64-bit one over what the caches stand for, and the caches hold what was packed."""
    b, hq, hkv, d, cap, n = 2, 8, 2, 128, 90, 60
    bk = ga._bk(b, hq, hkv, d, cap, n_beacons=0, window=4, n_prefix=2)
    K4, V4, S4 = new_cache(b, hkv, cap, d=d)
    w = torch.zeros(b, hkv, cap, device=DEV)
    length = ga._lens(b, hkv, [n, n - 7, 31, n])
    K, V = rows(b, hkv, n, d, seed=1), rows(b, hkv, n, d, seed=2)
    try:
        bk.reserve_attend4(n_q=1, weights=True)
        bk.pack4(K, V, K4, V4, S4, length=length)
        for step in range(70):
            if int(length.max()) == cap:
                kept, length = bk.evict4(K4[None], V4[None], S4[None], w[None], L=length[None].contiguous(), budget=50)
                length = length[0]
            k, v = rows(b, hkv, 1, d, seed=100 + step), rows(b, hkv, 1, d, seed=200 + step)
            before, length = length, length + 1
            bk.pack4(k, v, K4, V4, S4, first=before, length=length)
            q = rows(b, hq, 1, d, seed=300 + step)
            w0 = w.clone()
            o, lse = bk.attend4(q, K4, V4, S4, length=length, weights=w)
            bk.sync()
            at = before.long()
            for x in range(b):
                for y in range(hkv):
                    assert torch.equal(K4[x, y, at[x, y]], to_words(pack64(k[x, y, 0])[0], 0))
            if step % 9 == 0:
                (o64, l64, w64), (to, tl, tw) = reference4(q, K4, V4, S4, length)
                ga.check(o, o64, to, "o")
                ga.check(lse, l64, tl, "lse")
                ga.check(w, w0.double() + w64, tw + 2.0 ** -23 * (w0 + w64), "weights")
    finally:
        bk.close()


@pytest.mark.parametrize("n_q", [1, 30])
def test_captured_and_replayed(n_q):
    """A step of packing and attention captured into a graph, replayed with other contents of the same buffers; a larger
    reservation in between leaves the graph its workspace."""
    b, hq, hkv, d, cap = 2, 8, 2, 64, 400
    st = torch.cuda.Stream()
    lens = ga._lens(b, hkv, [400, 333, 64, 399])
    first = lens - n_q
    q, (K4, V4, S4) = case(b, hq, hkv, d, cap, n_q, lens)
    k, v = rows(b, hkv, n_q, d, seed=1), rows(b, hkv, n_q, d, seed=2)
    bk = ga._bk(b, hq, hkv, d, cap, stream=st)
    try:
        bk.reserve_attend4(n_q=n_q)
        o, lse = torch.zeros_like(q), torch.zeros(b, hq, n_q, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            bk.pack4(k, v, K4, V4, S4, first=first, length=lens)
            bk.attend4(q, K4, V4, S4, length=lens, o_out=o, lse_out=lse)
        bk.reserve_attend4(n_q=64, weights=True)
        for seed in (7, 8):
            k.copy_(rows(b, hkv, n_q, d, seed=seed))
            q.copy_(rows(b, hq, n_q, d, seed=seed + 10))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want, want_l = bk.attend4(q, K4, V4, S4, length=lens)
            bk.sync()
            assert torch.equal(o, want) and torch.equal(lse, want_l)
            for x in range(b):
                for y in range(hkv):
                    f = int(first[x, y])
                    assert torch.equal(K4[x, y, f:f + n_q], to_words(pack64(k[x, y])[0], 0))
    finally:
        bk.close()
