"""4-bit caches at the ends of their numbers' ranges.  References and tolerances are those of
tests/test_gpu_four_bit.py where nothing else is said."""
import math

import pytest
import torch

from tests import test_gpu_attend as ga
from tests import test_gpu_four_bit as fb

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("d", [64, 128])
def test_elements_past_the_range_of_low_and_step(d):
    """Low and step are limited, not the elements: what larger ones stand for, and that bf16 elements up to 65280, the
    last below 65504, stand for numbers below it."""
    def group(*x):
        return torch.tensor(x, device=DEV).repeat(32 // len(x))

    top = 65504.0
    rows = torch.stack([torch.cat([g] * (d // 32)) for g in (
        group(3e38, 3e38), group(-3e38, -3e38), group(0.0, 1e5), group(-3e38, 3e38), group(0.0, 3e38),
        group(-65280.0, 65280.0), group(-65280.0, 64768.0), group(-256.0, 65280.0))]).bfloat16()
    K = rows[None, None].contiguous()
    n = K.shape[2]
    lens = ga._lens(1, 1, [n])
    bk = ga._bk(1, 1, 1, d, n)
    try:
        K4, V4, S4 = fb.new_cache(1, 1, n, d=d)
        bk.pack4(K, K, K4, V4, S4, length=lens)
        bk.sync()
        for which, words in enumerate((K4, V4)):
            v = fb.values64(words, S4, which)[0][0, 0]
            assert bool((v[0] == 16 * top).all())                       # a constant group: low + 15 step
            assert bool((v[1] == -top).all())
            assert bool((v[2, 1::2] - 1e5).abs().max() <= 1e5 * 2.0 ** -8) and bool((v[2, ::2] == 0).all())
            assert bool((v[3, 1::2] == 14 * top).all()) and bool((v[3, ::2] == -top).all())
            assert bool((v[4, 1::2] == 15 * top).all()) and bool((v[4, ::2] == 0).all())
            assert bool((v[5:].abs() <= top).all())
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q,weights", [(2, 60, True), (1, 150, True), (4, 40, False)])
def test_queries_of_every_magnitude_in_calls_of_many_rows(d, G, n_q, weights):
    """Rows of queries times powers of two, with scales to match, within one call and from call to call.  Multiplied by
    2^k, with the scale divided by it, a query is the same, so the reference is that of the queries as they were (whose
    2^-25 for small elements, at most 2^-39 of a row's largest now, is 2^-10 of what a logit may be off by)."""
    b, hkv, cap = 2, 2, 400
    lens = ga._lens(b, hkv, [400, 301, 129, 170])
    q, cache = fb.case(b, G * hkv, hkv, d, cap, n_q, lens, seed=n_q)
    q[:, 0, ::3, 1:] *= 2.0 ** -20          # one element far above the others
    q[:, 1, 1::3] = 0
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    scale = 1 / math.sqrt(d)

    try:
        ref = fb.reference4(q, *cache, lens, many=True)
        for power in (-60, -30, 60):
            qq = (q.double() * 2.0 ** power).bfloat16()
            fb.run4(bk, qq, cache, lens, weights=weights, scale=scale * 2.0 ** -power, ref=ref)
        # of one call, every second head's rows times 2^20 or 2^-40
        for power in (20, -40):
            qq = q.clone()
            qq[:, ::2] = (q[:, ::2].double() * 2.0 ** power).bfloat16()
            K4, V4, S4 = cache
            bk.reserve_attend4(n_q=n_q)
            o, lse = bk.attend4(qq, K4, V4, S4, length=lens, scale=scale * 2.0 ** -power)
            bk.sync()
            (o64, l64, _), (to, tl, _) = ref
            ga.check(o[:, ::2], o64[:, ::2], to[:, ::2], "o")
            ga.check(lse[:, ::2], l64[:, ::2], tl[:, ::2], "lse")
    finally:
        bk.close()


def weighted(b, hkv, cap, d, far, V, seed=0):
    """Caches whose keys have weights by design with queries of ones and the scale ln 2 / d: of every 16 keys 2^0 for one,
    2^-60 for one, 2^far for the others (rows of one value, exact in fp16); V holds what the test gives it."""
    y = torch.full((b, hkv, cap), float(far), device=DEV)
    y[:, :, 3::16] = -60.0
    y[:, :, 5::16] = 0.0
    return fb.packed(y[..., None].expand(b, hkv, cap, d).bfloat16(), V.bfloat16())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(4, 1), (3, 4)])
@pytest.mark.parametrize("what", ["a large row", "large rows", "a large group", "small values", "both"])
def test_values_of_many_small_weights(d, G, n_q, what):
    """Keys with zeros as values have all the weight, of the others each 2^-22 of one of these: what they add up to is the
    output.  Large rows of no weight, a large group of elements and values near fp16's smallest do not take their digits.
    |o - o64| is as in tests/test_gpu_four_bit.py but for what fp16 rounds below its normal range: p stands as p 2^11
    against a reference of the row's largest at most, off by 2^-36 of that, of a low; a product of it and a step of
    2^-11 to 1 by as much, or any by 2^-33 of the largest such product, each times a code of 15 at most."""
    b, hkv, cap = 1, 2, 20011
    lens = ga._lens(b, hkv, [cap, 19000])
    g = torch.Generator(device=DEV).manual_seed(d + G)
    V = torch.rand(b, hkv, cap, d, generator=g, device=DEV) + 0.5
    if what == "a large row":
        V[:, :, 3] = 60000 * torch.sign(torch.randn(d, generator=g, device=DEV))
    if what in ("large rows", "both"):
        V[:, :, 3::16] *= 40000.0 * torch.sign(torch.randn(d, generator=g, device=DEV))
    if what in ("a large group", "both"):
        V[..., :32] = (V[..., :32] - 0.9) * 50000
    if what == "small values":
        V *= 2.0 ** -16
    if what == "both":
        V[..., 32:] *= 2.0 ** -12
    V[:, :, 5::16] = 0
    cache = weighted(b, hkv, cap, d, -22, V)
    fb.poison(cache, lens)
    scale = math.log(2.0) / d
    q = torch.ones(b, G * hkv, n_q, d, device=DEV).bfloat16()
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        _, lse, _ = fb.run4(bk, q, cache, lens, scale=scale)
        o, _ = bk.attend4(q, *cache, length=lens, scale=scale)
        bk.sync()
        (o64, l64, _), _ = fb.reference4(q, *cache, lens, scale)
        for y in range(hkv):
            n = int(lens[0, y])
            _, k_sn, k_low = fb.values64(cache[0][0, y, :n], cache[2][0, y, :n], 0)
            v, sn, low = fb.values64(cache[1][0, y, :n], cache[2][0, y, :n], 1)
            step = cache[2][0, y, :n, 1, :, 0].double().repeat_interleave(32, -1)
            ordinary = ((step >= 2.0 ** -11) & (step <= 1)).any(0)
            for i in range(n_q):
                m = n - n_q + 1 + i
                z = k_low[:m, 0] * d * scale
                p = torch.exp(z - torch.logsumexp(z, 0))
                delta = 2 * 2.0 ** -16 * float(k_low[:m, 0].abs().max()) * math.log(2.0) + 2.0 ** -14
                off = ((2.0 ** -10 + 2 * delta) * (p @ sn[:m]) + (2.0 ** -11 + 2 * delta) * (p @ low[:m].abs())
                       + 2.0 ** -36 * p.max() * (15 * m * ordinary + low[:m].abs().sum(0))
                       + 15 * m * 2.0 ** -33 * (p[:, None] * step[:m]).amax(0))
                want = p @ v[:m]
                for h in range(y * G, (y + 1) * G):
                    ga.check(o[0, h, i], want, 2.0 ** -8 * want.abs() + off, f"o of {what}")
    finally:
        bk.close()


@pytest.mark.parametrize("d,G,n_q,weights,many", [
    (128, 3, 16, True, False), (128, 7, 7, True, True), (64, 16, 3, True, False), (64, 7, 7, True, True),
    (128, 8, 12, False, False), (128, 1, 97, False, True), (64, 5, 16, False, False), (64, 1, 81, False, True)])
def test_rows_on_both_sides_of_a_border(d, G, n_q, weights, many):
    """48 and 49 rows with weights, 96 and 97 without (80 and 81 of head_dim 64): the last that are read code by code, and
    the first that are read unpacked."""
    b, hkv, cap = 2, 2, 500
    lens = ga._lens(b, hkv, [500, 257, 128, 33])
    q, cache = fb.case(b, G * hkv, hkv, d, cap, n_q, lens, seed=n_q)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        fb.run4(bk, q, cache, lens, weights=weights, ref=fb.reference4(q, *cache, lens, many=many))
    finally:
        bk.close()
