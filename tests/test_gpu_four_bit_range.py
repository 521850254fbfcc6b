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
