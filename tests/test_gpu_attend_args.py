"""Arguments that share memory, workspaces that graphs hold, and what an eviction refuses."""
import math

import pytest
import torch

from paper_2609_04971_gb300 import bkv
from tests.test_gpu_attend import _bk, _inputs, _lens, check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q", [2, 40])
def test_overlapping_arguments_are_refused(n_q):
    """Every output is written while inputs may still be read; none may share a byte with an input or another."""
    b, hq, hkv, d, cap = 4, 4, 2, 64, 100
    q, K, V = _inputs(b, hq, hkv, d, cap, n_q, seed=31)
    lens = _lens(b, hkv, [100])
    Kp, Vp = K[:2].clone(), V[:2].clone()
    pl = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 3.0), torch.full((b, hq, n_q), 3.0, device="cuda")
    w = torch.full((b, hkv, cap), 3.0, device="cuda")
    before = [t.clone() for t in (q, K, V, Kp, Vp, lens, pl, o, lse, w)]
    bk = _bk(b, hq, hkv, d, cap)

    def refused(shared=False, **kw):
        a = dict(q=q, K=K, V=V, length=lens, Kp=Kp, Vp=Vp, prefix_len=pl, o=o, lse=lse, w=w)
        a.update(kw)
        with pytest.raises(bkv.BkvError) as ei:
            if shared:
                bkv.bkv_attend_shared(bk.ctx, a["q"], n_q, a["Kp"], a["Vp"], a["prefix_len"], 2, cap, a["K"], a["V"],
                                      a["length"], 0.0, a["o"], a["lse"], a["w"])
            else:
                bkv.bkv_attend(bk.ctx, a["q"], n_q, a["K"], a["V"], a["length"], 0.0, a["o"], a["lse"], a["w"])
        assert ei.value.code == bkv.BKV_EINVAL

    def view(t, dtype, at=0):  # another type's view of the last bytes of t, or of those `at` bytes from its start
        return t.view(-1).view(torch.uint8)[at:].view(dtype)

    try:
        bk.reserve_attend(n_q=n_q, n_groups=2, weights=True)
        for shared in (False, True):
            refused(shared, o=q)
            refused(shared, o=view(q, torch.bfloat16, 16))   # shifted by 16 bytes
            refused(shared, o=K)
            refused(shared, o=V)
            refused(shared, o=view(w, torch.bfloat16))
            refused(shared, o=view(lse, torch.bfloat16))
            refused(shared, lse=view(q, torch.float32))
            refused(shared, lse=view(K, torch.float32))
            refused(shared, lse=view(lens, torch.float32))
            refused(shared, lse=w)
            refused(shared, w=view(V, torch.float32))
            refused(shared, w=view(q, torch.float32, q.numel() * 2 - 4))  # one element
            refused(shared, w=view(lens, torch.float32))
        refused(True, o=Kp)
        refused(True, o=Vp)
        refused(True, lse=view(pl, torch.float32))
        refused(True, w=view(Kp, torch.float32))
        bk.sync()
        for x, y in zip((q, K, V, Kp, Vp, lens, pl, o, lse, w), before):
            assert torch.equal(x, y)
        # inputs may share memory with one another, and outputs may lie side by side
        room = torch.zeros(q.numel() * 2 + 4 * lse.numel() + 4 * w.numel(), dtype=torch.uint8, device="cuda")
        n1, n2 = q.numel() * 2, q.numel() * 2 + 4 * lse.numel()
        o2, l2, w2 = (room[:n1].view(torch.bfloat16).view(q.shape), room[n1:n2].view(torch.float32).view(lse.shape),
                      room[n2:].view(torch.float32).view(w.shape))
        bkv.bkv_attend(bk.ctx, q, n_q, K, K, lens, 0.0, o2, l2, w2)
        want, want_l = bk.attend(q, K, K.clone(), length=lens)
        bk.sync()
        assert torch.equal(o2, want) and torch.equal(l2, want_l) and bool((w2.sum(-1) > 0).all())
    finally:
        bk.close()


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


def test_a_graph_outlives_a_larger_reservation():
    """A decode step is captured, then a prompt reserves more: the graph's workspace stays its own, so that neither
    the allocator's next tensors nor calls in the new workspace reach it."""
    b, hq, hkv, d, cap = 2, 8, 2, 128, 6000
    q, K, V = _inputs(b, hq, hkv, d, cap, 1, seed=10)
    qp, Kp, Vp = _inputs(b, hq, hkv, d, cap, 300, seed=11)
    lens, lens_p = _lens(b, hkv, [6000, 5, 200, 5128]), _lens(b, hkv, [300, 4000, 900, 301])
    w = torch.zeros(b, hkv, cap, device="cuda")
    o = torch.empty(b, hq, 1, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(b, hq, 1, device="cuda")
    (o64, l64, w64), (to, tl, tw) = reference(q, K, V, lens)
    (op64, lp64, _), (top, tlp, _) = reference(qp, Kp, Vp, lens_p)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    bk = _bk(b, hq, hkv, d, cap, stream=stream)
    free = lambda: torch.cuda.mem_get_info()[0]  # noqa: E731
    try:
        with torch.cuda.stream(stream):
            bk.reserve_attend(weights=True)
            bk.attend(q, K, V, length=lens, weights=w, o_out=o, lse_out=lse)
            bk.sync()
            graphs = []
            for n_q in (None, 64, 300):  # each reservation is larger than the one before
                if n_q:
                    bk.reserve_attend(n_q=n_q, weights=True)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    bk.attend(q, K, V, length=lens, weights=w, o_out=o, lse_out=lse)
                graphs.append(graph)
            junk = [torch.full((n,), math.nan, device="cuda") for n in [1 << 20] * 8 + [1 << 22] * 4]
            for graph in graphs:
                for t in (o, lse, w):
                    t.fill_(math.nan if t is not w else 0)
                op, lp = bk.attend(qp, Kp, Vp, length=lens_p)
                graph.replay()
                bk.sync()
                check(o, o64, to, "o")
                check(lse, l64, tl, "lse")
                check(w, w64, tw, "weights")
                check(op, op64, top, "o of the prompt")
                check(lp, lp64, tlp, "lse of the prompt")
            assert all(bool(t.isnan().all()) for t in junk)
            del graphs, graph
        torch.cuda.synchronize()
        before = free()
    finally:
        bk.close()
    assert free() > before  # all workspaces, the old ones among them


@pytest.mark.parametrize("cap", [300, 5000, 12000])
def test_refused_instances_are_untouched(cap):
    """Lengths out of range among good ones: kept rows -1, new length 0, and nothing else of the instance written,
    in place and into another cache."""
    shape, d, budget = (1, 2, 3), 64, 120
    K, V = (torch.randn(*shape, cap, d, device="cuda").bfloat16() for _ in "KV")
    w = torch.rand(*shape, cap, device="cuda")
    L = torch.tensor([cap + 1, cap, -1, 121, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda").view(shape)
    bad = [0, 2, 4, 5]
    bk = _bk(2, 3, 3, d, cap, window=8, n_beacons=0, n_prefix=2)
    try:
        for in_place in (True, False):
            rows = cap if in_place else budget
            Ko, Vo, wo = (K.clone(), V.clone(), w.clone()) if in_place else (
                torch.randn(*shape, rows, d, device="cuda").bfloat16(),
                torch.randn(*shape, rows, d, device="cuda").bfloat16(), torch.full((*shape, rows), 7.0, device="cuda"))
            before = [t.clone() for t in (Ko, Vo, wo)]
            src = (Ko, Vo, wo) if in_place else (K, V, w)
            kept, new = bk.evict(*src, L=L, budget=budget, K_out=Ko, V_out=Vo, weights_out=wo)
            with pytest.raises(bkv.BkvError) as ei:
                bk.sync()
            assert ei.value.code == bkv.BKV_EINVAL
            bk.sync()
            flat = lambda t: t.flatten(0, 2)  # noqa: E731
            assert new.flatten().tolist() == [0, budget, 0, budget, 0, 0]
            for e in bad:
                assert bool((flat(kept)[e] == -1).all())
                for x, y in zip((Ko, Vo, wo), before):
                    assert torch.equal(flat(x)[e], flat(y)[e])
            for e in (1, 3):
                at = flat(kept)[e].long()
                assert bool((at[1:] > at[:-1]).all())
                for x, y in zip((Ko, Vo, wo), (K, V, w)):
                    assert torch.equal(flat(x)[e, :budget], flat(y)[e, at])
    finally:
        bk.close()


@pytest.mark.parametrize("G,window", [(8, 32), (16, 64), (1, 64)])
def test_windows_past_the_scoring_limit(G, window):
    """G * window is bounded by a compress's scoring queries.  Eviction does not see query heads: a context with as
    many query heads as KV heads takes every window up to 64."""
    with pytest.raises(bkv.BkvError):
        _bk(2, 2 * 64, 2, 64, 200, window=window, n_beacons=0)  # 64 query heads to a KV head
    b, hkv, d, cap, budget = 2, 2, 64, 200, 100
    shape = (1, b, hkv)
    K, V = (torch.randn(*shape, cap, d, device="cuda").bfloat16() for _ in "KV")
    w = torch.zeros(*shape, cap, device="cuda")
    lens = torch.full(shape, cap, dtype=torch.int32, device="cuda")
    q = torch.randn(b, G * hkv, 1, d, device="cuda").bfloat16()
    att, ev = _bk(b, G * hkv, hkv, d, cap), _bk(b, hkv, hkv, d, cap, window=window, n_beacons=0)
    try:
        att.reserve_attend(weights=True)
        att.attend(q, K[0], V[0], length=lens[0], weights=w[0])
        att.sync()
        kept, new = ev.evict(K, V, w, L=lens, budget=budget)
        ev.sync()
        assert bool((new == budget).all())
        assert bool((kept[..., -window:] == torch.arange(cap - window, cap, device="cuda")).all())
    finally:
        att.close()
        ev.close()
