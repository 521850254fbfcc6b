"""Attention whose blocks take several key tiles each, in row blocks that rows do not fill, and merges of many parts;
values against the 64-bit reference and with the tolerances of test_gpu_attend."""
import math

import pytest
import torch

from tests.test_gpu_attend import _bk, _inputs, _lens, _poison, run_and_check

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
