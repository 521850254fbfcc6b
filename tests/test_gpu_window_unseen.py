"""Rows that no query sees through a window may hold anything, as rows past a length may: they share a block of 128 rows
with a first key that stays visible, or lie before every window."""
import math

import pytest
import torch

from tests import test_gpu_attend as ga
from tests import test_gpu_window as gw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(4, 1), (3, 5), (2, 40), (1, 140), (4, 64), (2, 300)])
@pytest.mark.parametrize("window,n_sink", [(90, 4), (150, 20), (60, 130), (200, 0), (1, 1)])
def test_nothing_of_unseen_rows_matters(d, G, n_q, window, n_sink):
    b, hkv, cap = 2, 2, 700
    lens = ga._lens(b, hkv, [700, 230, window + n_q + 30, 161])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, n_q, seed=n_q)
    for x in range(b):
        for y in range(hkv):
            n = int(lens[x, y])
            first = max(n_sink, n - n_q + 1 - window, 0)  # what the first query's window reaches
            for z, bad in enumerate((math.nan, math.inf, -math.inf)):
                K[x, y, n_sink:first][z::3], V[x, y, n_sink:first][z::3] = bad, -bad
                K[x, y, n:][z::3], V[x, y, n:][z::3] = -bad, bad
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        bk.reserve_attend(n_q=n_q)
        o, lse = bk.attend_window(q, K, V, length=lens, window=window, n_sink=n_sink)
        bk.sync()
        K0, V0 = (torch.where(t.isfinite(), t, 0.0) for t in (K, V))
        (o64, l64), (to, tl) = gw.reference(q, K0, V0, lens, window, n_sink)
        ga.check(lse, l64, tl, "lse")
        ga.check(o, o64, to, "o")
    finally:
        bk.close()
