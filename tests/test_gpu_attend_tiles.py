"""Attention whose blocks take several key tiles each, in row blocks that rows do not fill, and merges of many parts;
values against the 64-bit reference and with the tolerances of test_gpu_attend."""
import math

import pytest
import torch

from tests.test_gpu_attend import _bk, _inputs, _lens, _poison, check, reference, run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("groups,m,G,n_q", [(2, 3, 4, 25), (3, 5, 4, 25), (2, 5, 8, 8), (2, 2, 4, 70), (4, 3, 1, 90)])
def test_uneven_row_blocks_of_several_groups(d, groups, m, G, n_q):
    """More than 128 rows per prefix in blocks that the number of sequences does not fill; logits of +-35, so that
    references move and a row of the next group would move them too."""
    b, hkv, cap, pcap = groups * m, 4, 260, 1500
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=m, std=8.0)
    _, Kp, Vp = _inputs(groups, 1, hkv, d, pcap, 1, seed=m + 1)
    lens = _lens(b, hkv, [0, 1, 129, 260, 128, 17, 40])
    pl = torch.tensor([1500, 1281, 700, 0][:groups], dtype=torch.int32, device="cuda")
    _poison(K, V, lens)
    _poison(Kp, Vp, pl[:, None].expand(groups, hkv))
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens, Kp=Kp, Vp=Vp, plens=pl)
        run_and_check(bk, q, K, V, lens, Kp=Kp, Vp=Vp, plens=pl, weights=False)
    finally:
        bk.close()


def test_time_does_not_depend_on_another_group():
    """Three sequences of 100 rows in row blocks of two: the second block's other half is filled with the next
    group's queries, whose rows are not used.  What those queries are must not show in the time.  They see only
    zero keys in their own prefix, so their own block does the same work whatever they are."""
    groups, m, G, n_q, hkv, d, pcap, cap = 2, 3, 4, 25, 8, 128, 16384, 64
    b = groups * m
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=1, std=0.1)
    _, Kp, Vp = _inputs(groups, 1, hkv, d, pcap, 1, seed=2)
    unit = torch.ones(d, device="cuda") / math.sqrt(d)
    Kp[0] = (40 * unit + 0.1 * Kp[0].float()).bfloat16()
    Kp[1] = 0
    K.zero_()
    lens = _lens(b, hkv, [n_q])
    plens = torch.tensor([pcap, pcap], dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(b, G * hkv, n_q, device="cuda")
    bk = _bk(b, G * hkv, hkv, d, cap)

    def time(other):
        q[m:] = other
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = math.inf
        for _ in range(6):
            start.record()
            for _ in range(10):
                bk.attend_shared(q, Kp, Vp, K, V, prefix_len=plens, length=lens, o_out=o, lse_out=lse)
            stop.record()
            stop.synchronize()
            best = min(best, start.elapsed_time(stop))
        return best

    try:
        bk.reserve_attend(n_q=n_q, n_groups=groups)
        zero, large = time(0.0), time(1.0)  # logits of 0, and of 40, against the first group's keys
        bk.sync()
        print(f"{zero * 100:.1f} and {large * 100:.1f} us a call")
        assert large < 1.2 * zero
    finally:
        bk.close()


def _tiles_per_block(items, tiles):
    """Key tiles of a block of the attention kernels, one block to an SM, when every item has `tiles`."""
    return items * tiles / torch.cuda.get_device_properties(0).multi_processor_count


def _run_and_check_wide(bk, q, K, V, lens, weights):
    """run_and_check for logits that span more than the exponents of fp32: a term of a weight's sum below 2^-126 may
    count as 0, so each of the R terms adds 2^-126 to the tolerance of the sum (no fp32 number is as near as 2^-24 of
    itself to a sum of 10^-138)."""
    R = q.shape[1] // K.shape[1] * q.shape[2]
    w0 = torch.rand(*K.shape[:3], device="cuda")
    w = w0.clone() if weights else None
    bk.reserve_attend(n_q=q.shape[2], weights=weights)
    o, lse = bk.attend(q, K, V, length=lens, weights=w)
    bk.sync()
    (o64, l64, w64), (to, tl, tw) = reference(q, K, V, lens)
    check(lse, l64, tl, "lse")
    check(o, o64, to, "o")
    if weights:
        past = torch.arange(K.shape[2], device="cuda") >= lens[..., None]
        assert torch.equal(w[past], w0[past])
        check(w, w0.double() + w64, tw + 2.0 ** -23 * (w0 + w64) + R * 2.0 ** -126, "weights")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["rising", "falling", "steps", "mixed", "late"])
@pytest.mark.parametrize("n_q", [1, 4, 12, 20, 32, 60, 64])
def test_reference_moves_within_a_segment(order, n_q, d):
    """Caches of twelve tiles, five of them to a block: logits that rise by more than 2^32 from tile to tile (in
    some rows only; late in a tile; by steps) move a block's references when it has sums and outputs to scale.  A
    move multiplies them by a factor that is off by 2^-22, at most twelve times: well within the 2^-14 that the
    reference allows an exponential."""
    b, G, hkv, cap = 8, 4, 8, 1500
    assert _tiles_per_block(b * hkv, 12) > 4
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=13, std=1.0)
    unit = torch.ones(d, device="cuda") / math.sqrt(d)
    j = torch.arange(cap)
    level = {"rising": torch.linspace(-150, 150, cap), "falling": torch.linspace(150, -150, cap),
             "steps": (j // 300) * 40.0, "mixed": torch.linspace(-100, 200, cap),
             "late": torch.where(j % 128 == 127, (j // 128) * 30.0, -20.0)}[order].cuda()
    q[:] = (unit * math.sqrt(d) + 0.02 * q).bfloat16()  # q . k / sqrt(d) = level + noise
    if order == "mixed":  # half of the rows fall while the others rise
        q[:, ::2] = -q[:, ::2]
    K[:] = (level[:, None] * unit + 0.1 * K).bfloat16()
    lens = _lens(b, hkv, [1500, 1400, 1450, 1281, 1500, 900])
    _poison(K, V, lens)
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        _run_and_check_wide(bk, q, K, V, lens, True)
        _run_and_check_wide(bk, q, K, V, lens, False)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,G", [(1, 4), (1, 16), (2, 8), (5, 4), (6, 4), (11, 4), (16, 4), (20, 4), (23, 4), (28, 4),
                                   (32, 4), (130, 1), (40, 4), (64, 4), (75, 4), (200, 3)])
def test_several_tiles_per_block(d, n_q, G):
    """Every column count of the kernel with keys as lanes, then rows as lanes in one and in two row blocks."""
    b, hkv, cap = 8, 8, 1400
    assert _tiles_per_block(b * hkv, 11) > 4
    lens = _lens(b, hkv, [1400, 1399, 1280, 0, 1153, 700, 1, 129, 1281])
    q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=n_q)
    _poison(K, V, lens)
    bk = _bk(b, G * hkv, hkv, d, cap)
    try:
        run_and_check(bk, q, K, V, lens)
        run_and_check(bk, q, K, V, lens, weights=False)
    finally:
        bk.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q,G", [(11, 4), (25, 4), (40, 4), (100, 4)])
def test_one_long_cache_among_many(d, n_q, G):
    """Its rows come in some sixty parts, many more than a pass over the parts takes at once, beside items that one
    block finishes."""
    b, hkv, cap = 20, 2, 8300
    for values in ([8300] + [130] * 39, [60, 8299] + [1] * 20 + [0] * 17 + [8300]):
        lens = _lens(b, hkv, values)
        q, K, V = _inputs(b, G * hkv, hkv, d, cap, n_q, seed=70)
        _poison(K, V, lens)
        bk = _bk(b, G * hkv, hkv, d, cap)
        try:
            run_and_check(bk, q, K, V, lens)
            run_and_check(bk, q, K, V, lens, weights=False)
        finally:
            bk.close()


@pytest.mark.parametrize("groups", [0, 2])
def test_values_within_one_reservation(groups):
    """Calls of several sizes in the workspace of the largest: its regions move with the size."""
    b, hq, hkv, d, cap = 4, 8, 2, 64, 12000
    lens = _lens(b, hkv, [700, 333, 0, 12000])
    bk = _bk(b, hq, hkv, d, cap)
    try:
        bk.reserve_attend(n_q=300, n_groups=groups, weights=True)
        for n_q in (300, 1, 257, 8, 33, 9, 64, 300):
            q, K, V = _inputs(b, hq, hkv, d, cap, n_q, seed=n_q)
            _poison(K, V, lens)
            kw = {}
            if groups:
                Kp, Vp = _inputs(groups, hq, hkv, d, 150, 1, seed=51)[1:]
                kw = dict(Kp=Kp, Vp=Vp, plens=torch.tensor([150, 0], dtype=torch.int32, device="cuda"))
            run_and_check(bk, q, K, V, lens, **kw)
    finally:
        bk.close()
