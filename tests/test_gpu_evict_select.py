"""Selection of the evicted rows where many weights share their leading bits: the kept rows are those of a sort."""
import pytest
import torch

from tests.test_gpu_attend import _bk, evict_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cap,shared", [
    (1500, 1), (1501, 128), (1500, 129), (1500, 640), (1500, 641), (1502, 1502),
    (5000, 128), (5003, 1280), (5000, 1281), (5000, 5000),
    (12000, 129), (12000, 2560), (12001, 2561), (32768, 32768),
])
@pytest.mark.parametrize("step", [0, 1, 1500])
@pytest.mark.parametrize("offset", [0, 1])
def test_weights_with_common_leading_bits(cap, shared, step, offset):
    """`shared` weights of [1, 1.125), `step` units in the last place apart and five of each; the others are spread on
    both sides of them.  The last kept row is one of them: the first, one in the middle, the last.  The weights begin
    at a multiple of 16 bytes or 4 bytes behind one."""
    g = torch.Generator().manual_seed(cap + shared)
    lens = (cap, cap - 1)
    w = torch.empty(1, 1, 2, cap)
    n_above = (cap - shared) // 2
    for e in range(2):
        mid = (torch.arange(shared, dtype=torch.int32) // 5 * step % (1 << 20) + 0x3F800000).view(torch.float32)
        above, below = 1.125 + torch.rand(n_above, generator=g), torch.rand(cap - shared - n_above, generator=g)
        w[0, 0, e] = torch.cat([mid, above, below])[torch.randperm(cap, generator=g)]
    w_dev = torch.empty(2 * cap + offset, device="cuda")[offset:].view(1, 1, 2, cap).copy_(w)
    L = torch.tensor(lens, dtype=torch.int32).view(1, 1, 2)
    K, V = (torch.randn(1, 1, 2, cap, 64, generator=g).bfloat16().cuda() for _ in "KV")
    bk = _bk(1, 2, 2, 64, cap, window=8, n_beacons=0, n_prefix=3)
    try:
        for k_sel in sorted({max(1, n_above), n_above + 1, n_above + shared // 2 + 1, cap - 12}):
            budget = min(k_sel, cap - 12) + 11
            w_out = torch.full((1, 1, 2, budget + 2), 7.0, device="cuda")
            K_out, V_out = (torch.zeros(1, 1, 2, budget + 2, 64, dtype=torch.bfloat16, device="cuda") for _ in "KV")
            kept, new = bk.evict(K, V, w_dev, L=L.cuda(), budget=budget, K_out=K_out, V_out=V_out, weights_out=w_out)
            bk.sync()
            for e, n in enumerate(lens):
                want = evict_reference(w[0, 0, e].tolist(), n, budget, 3, 8)
                assert new[0, 0, e].item() == len(want)
                assert kept[0, 0, e].tolist() == want + [-1] * (budget - len(want)), (budget, e)
                assert torch.equal(w_out[0, 0, e, :len(want)].cpu(), w[0, 0, e, want])
                assert bool((w_out[0, 0, e, len(want):] == 0).all())
                assert torch.equal(K_out[0, 0, e, :len(want)], K[0, 0, e, want])
    finally:
        bk.close()
