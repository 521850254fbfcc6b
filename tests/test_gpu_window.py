"""bkv_attend_window against a plain implementation in 64 bits.  The arithmetic is bkv_attend's, so are the tolerances
(tests/test_gpu_attend.py), with sums over the keys that a row sees."""
import math

import pytest
import torch

from paper_2609_04971_gb300 import bkv
from tests import test_gpu_attend as ga

pytestmark = pytest.mark.gpu


def reference(q, K, V, lens, window, n_sink, scale=None):
    b, hq, n_q, d = q.shape
    hkv = K.shape[1]
    G = hq // hkv
    scale = scale or 1 / math.sqrt(d)
    o = torch.zeros(b, hq, n_q, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq, n_q), -math.inf, dtype=torch.float64, device="cuda")
    to, tl = torch.zeros_like(o), torch.zeros_like(lse)
    for x in range(b):
        for y in range(hkv):
            n = int(lens[x, y])
            if n == 0:
                continue
            k, v = K[x, y, :n].double(), V[x, y, :n].double()
            j = torch.arange(n, device="cuda")[None]
            p_own = (n - n_q + torch.arange(n_q, device="cuda")).repeat(G)[:, None]
            seen = (j <= p_own) & ((j > p_own - window) | (j < n_sink))
            qq = q[x, y * G:(y + 1) * G].reshape(G * n_q, d).double()
            z = (qq @ k.T * scale).masked_fill(~seen, -math.inf)
            S = (qq.abs() @ k.abs().T * scale).masked_fill(~seen, 0).amax(-1)
            t = torch.logsumexp(z, -1)
            p = torch.exp(z - torch.where(t == -math.inf, 0.0, t)[:, None])
            delta = (2 * 2.0 ** -16 * S + 2.0 ** -14)[:, None]
            oo = p @ v
            r = slice(y * G, (y + 1) * G)
            o[x, r] = oo.view(G, n_q, d)
            to[x, r] = (ga.U * oo.abs() + (ga.U + 2 * delta) * (p @ v.abs())).view(G, n_q, d)
            lse[x, r] = t.view(G, n_q)
            tl[x, r] = (2.0 ** -16 * S + 2.0 ** -15 + 2.0 ** -22 * t.abs()).view(G, n_q)
    return (o, lse), (to, tl)


def run_and_check(bk, q, K, V, lens, window, n_sink, scale=None):
    bk.reserve_attend(n_q=q.shape[2])
    o, lse = bk.attend_window(q, K, V, length=lens, window=window, n_sink=n_sink, scale=scale)
    bk.sync()
    (o64, l64), (to, tl) = reference(q, K, V, lens, window, n_sink, scale)
    ga.check(lse, l64, tl, "lse")
    ga.check(o, o64, to, "o")
    return o, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 5, 17])
def test_single_tokens(d, G):
    """Windows and first keys around the tile borders and the small boxes of the first keys."""
    b, hkv, cap = 4, 2, 700
    lens = ga._lens(b, hkv, [1, 127, 128, 129, 700, 0, 255, 431])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, 1, seed=G)
    ga._poison(K, V, lens)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        for window in (1, 2, 100, 127, 128, 129, 300):
            for n_sink in (0, 1, 15, 16, 17, 130):
                run_and_check(bk, q, K, V, lens, window, n_sink)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(1, 2), (4, 5), (2, 40), (1, 128), (5, 25)])
def test_several_tokens(d, G, n_q):
    """Rows that begin to see keys at different places, windows and caches shorter than the new tokens."""
    b, hkv, cap = 3, 2, 520
    lens = ga._lens(b, hkv, [520, max(1, n_q - 1), n_q, 300, 131, 256])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, n_q, seed=n_q)
    ga._poison(K, V, lens)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        for window in (1, 7, 64, 128, 200):
            for n_sink in (0, 4, 140):
                run_and_check(bk, q, K, V, lens, window, n_sink)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,n_q", [(1, 129), (3, 300), (7, 33)])
def test_many_rows(d, G, n_q):
    b, hkv, cap = 2, 2, 1000
    lens = ga._lens(b, hkv, [1000, n_q + 3, n_q // 2, 641])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, n_q, seed=n_q)
    ga._poison(K, V, lens)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        for window, n_sink in ((1, 0), (1, 1), (5, 4), (128, 0), (128, 4), (129, 17), (256, 0), (256, 300), (500, 4)):
            run_and_check(bk, q, K, V, lens, window, n_sink)
    finally:
        bk.close()


@pytest.mark.parametrize("G,n_q", [(4, 1), (4, 17), (2, 200)])
@pytest.mark.parametrize("sign", [1, -1])
def test_keys_outside_the_window_do_not_matter(G, n_q, sign):
    """Logits of thousands on keys that some rows see and others do not: no row's reference may come from a key that
    it does not see.  sign < 0: the unseen ones lie thousands below."""
    b, hkv, d, cap = 2, 2, 64, 900
    lens = ga._lens(b, hkv, [900, 777, 513, 640])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, n_q, seed=3, std=1.0)
    u = torch.ones(d, device="cuda")
    q = (q.float() + u).bfloat16()
    steps = torch.arange(cap, device="cuda") // 50 % 7  # levels that change along the cache
    K = (K.float() + sign * 8.0 * steps[:, None] * u).bfloat16()
    K[:, :, :20] = (K[:, :, :20].float() + sign * 500.0 * u).bfloat16()
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        for window, n_sink in ((3, 0), (60, 0), (150, 0), (150, 4), (400, 0), (400, 30)):
            run_and_check(bk, q, K, V, lens, window, n_sink)
    finally:
        bk.close()


@pytest.mark.parametrize("G,n_q", [(4, 1), (3, 20), (2, 150)])
def test_a_window_that_holds_everything_is_plain_attention(G, n_q):
    b, hkv, d, cap = 2, 2, 128, 600
    lens = ga._lens(b, hkv, [600, 333, 128, 599])
    q, K, V = ga._inputs(b, G * hkv, hkv, d, cap, n_q, seed=1)
    bk = ga._bk(b, G * hkv, hkv, d, cap)
    try:
        bk.reserve_attend(n_q=n_q)
        want = bk.attend(q, K, V, length=lens)
        for window, n_sink in ((600, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 600)):
            got = bk.attend_window(q, K, V, length=lens, window=window, n_sink=n_sink)
            bk.sync()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    finally:
        bk.close()


@pytest.mark.parametrize("n_q", [1, 30])
def test_long_caches_in_parts_and_captured(n_q):
    """A few long caches whose windows many blocks share, on a stream of their own and out of a graph."""
    b, hq, hkv, d, cap = 1, 8, 2, 128, 20000
    st = torch.cuda.Stream()
    lens = ga._lens(b, hkv, [20000, 9001])
    q, K, V = ga._inputs(b, hq, hkv, d, cap, n_q, seed=4)
    bk = ga._bk(b, hq, hkv, d, cap, stream=st)
    try:
        bk.reserve_attend(n_q=n_q)
        torch.cuda.synchronize()
        o, lse = torch.zeros_like(q), torch.zeros(b, hq, n_q, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            bk.attend_window(q, K, V, length=lens, window=8192, n_sink=4, o_out=o, lse_out=lse)
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            want = run_and_check(bk, q, K, V, lens, 8192, 4)
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
            lens.copy_(ga._lens(b, hkv, [8193, 123]))
            torch.cuda.synchronize()
    finally:
        bk.close()


def test_refusals_and_lengths_out_of_range():
    b, hq, hkv, d, cap = 2, 4, 2, 64, 200
    lens = torch.tensor([[200, 201], [-1, 50]], dtype=torch.int32, device="cuda")
    ok = torch.tensor([[200, 0], [0, 50]], dtype=torch.int32, device="cuda")
    q, K, V = ga._inputs(b, hq, hkv, d, cap, 1)
    o = torch.empty_like(q)
    bk = ga._bk(b, hq, hkv, d, cap)
    try:
        with pytest.raises(bkv.BkvError) as ei:
            bk.attend_window(q, K, V, length=ok, window=8)
        assert ei.value.code == bkv.BKV_ESTATE
        bk.reserve_attend(n_q=1)
        for kw in (dict(window=0), dict(window=-5), dict(window=8, n_sink=-1), dict(window=8, scale=-1.0),
                   dict(window=8, o_out=q), dict(window=8, o_out=K.view(-1)[:q.numel()])):
            with pytest.raises(bkv.BkvError) as ei:
                bk.attend_window(q, K, V, length=ok, **kw)
            assert ei.value.code == bkv.BKV_EINVAL
        with pytest.raises(ValueError):
            bk.attend_window(q, K[:, :, :-1], V, length=ok, window=8)
        with pytest.raises(bkv.BkvError) as ei:
            bkv.bkv_attend_window(bk.ctx, q, 1, None, V, ok, 8, 0, 0.0, o)
        assert ei.value.code == bkv.BKV_EINVAL
        got = bk.attend_window(q, K, V, length=lens, window=60, n_sink=2)
        with pytest.raises(bkv.BkvError) as ei:
            bk.sync()
        assert ei.value.code == bkv.BKV_EINVAL
        want = bk.attend_window(q, K, V, length=ok, window=60, n_sink=2)
        bk.sync()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        bk.attend_window(q[:, :, :0], K, V, length=ok, window=60)
        bk.sync()
    finally:
        bk.close()
