"""4-bit caches at the ends of their numbers' ranges.  References and tolerances are those of
tests/test_gpu_four_bit.py where nothing else is said."""
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
