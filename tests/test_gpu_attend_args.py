"""Arguments that share memory, and eviction of instances whose length is refused."""
import pytest
import torch

from paper_2609_04971_gb300 import bkv
from tests.test_gpu_attend import _bk

pytestmark = pytest.mark.gpu


def test_overlapping_outputs_of_an_eviction_are_refused():
    """The kept rows and the new lengths are outputs like the others; only len_out may be L itself."""
    b, hkv, d, cap, budget = 2, 2, 64, 100, 50
    shape = (1, b, hkv)
    K, V = (torch.randn(*shape, cap, d, device="cuda").bfloat16() for _ in "KV")
    w = torch.rand(*shape, cap, device="cuda")
    L = torch.full(shape, cap, dtype=torch.int32, device="cuda")
    Ko, Vo = (torch.zeros(*shape, budget, d, dtype=torch.bfloat16, device="cuda") for _ in "KV")
    wo = torch.zeros(*shape, budget, device="cuda")
    kept = torch.full((*shape, budget), -7, dtype=torch.int32, device="cuda")
    new = torch.full(shape, -7, dtype=torch.int32, device="cuda")
    two = torch.full((2 * L.numel() - 1,), cap, dtype=torch.int32, device="cuda")
    tensors = (K, V, w, L, Ko, Vo, wo, kept, new, two)
    before = [t.clone() for t in tensors]
    bk = _bk(b, hkv, hkv, d, cap, window=8, n_beacons=0)

    def refused(in_place=False, L_=L, kept_=kept, new_=new):
        out = (K, V, w, cap) if in_place else (Ko, Vo, wo, budget)
        with pytest.raises(bkv.BkvError) as ei:
            bkv.bkv_evict(bk.ctx, K, V, w, L_, budget, *out, kept_, new_)
        assert ei.value.code == bkv.BKV_EINVAL

    i32 = lambda t: t.view(-1).view(torch.int32)  # noqa: E731
    try:
        for in_place in (False, True):
            refused(in_place, kept_=i32(w))
            refused(in_place, kept_=i32(K))
            refused(in_place, kept_=i32(V)[-1:])                 # reaches past V's end from its last element
            refused(in_place, kept_=L)
            refused(in_place, new_=kept)
            refused(in_place, new_=i32(w))
            refused(in_place, L_=two[:L.numel()], new_=two[L.numel() - 1:])  # one element of L
        refused(kept_=i32(wo))
        refused(kept_=i32(Ko))
        refused(new_=i32(wo)[-1:])
        refused(L_=i32(wo))
        bk.sync()
        for x, y in zip(tensors, before):
            assert torch.equal(x, y)
        bkv.bkv_evict(bk.ctx, K, V, w, L, budget, Ko, Vo, wo, budget, kept, L)
        bk.sync()
        assert bool((L == budget).all()) and bool((kept >= 0).all())
    finally:
        bk.close()
