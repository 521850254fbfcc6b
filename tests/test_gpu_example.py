"""The decoding example: without evictions it is the plain decoder; with them the caches stay in bounds."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_with_eviction.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decode_with_eviction", _PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _plain(m, prompt, first, fed):
    """The same model over whole sequences, attention in 64 bits: the prompt's last logits, and those after
    the tokens fed [n, samples] (the first of them `first`)."""
    out = []
    for seq in [prompt] + [torch.cat([prompt, fed[:, i]]) for i in range(first.numel())]:
        n = seq.numel()
        h, pos = m.embed[seq][None], torch.arange(n, device=seq.device)
        for layer in range(m.n_layers):
            q, k, v = m.project(layer, h, pos)
            G = m.n_q_heads // m.n_kv_heads
            k, v = k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
            z = q.double() @ k.transpose(-1, -2) / m.head_dim ** 0.5
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=seq.device).triu(1), -torch.inf)
            h = m.finish(layer, h, (z.softmax(-1) @ v).bfloat16())
        out.append(m.logits(h[:, -1])[0])
    return out[0], torch.stack(out[1:])


def test_without_evictions_it_is_the_plain_decoder(ex):
    """Budgets that hold everything.  The two differ by bf16 roundings of the attention output and what they
    become in two layers: outputs agree to a few units of 2^-8 of their size, logits (a sum of 512 terms of
    random sign, of unit size) to well below 2^-3."""
    m = ex.ToyModel()
    prompt = torch.randint(0, 512, (150,), generator=torch.Generator().manual_seed(3)).cuda()
    logits, Kp, Vp, plen = ex.run_prompt(m, prompt, 200)
    assert (plen == 150).all()
    first = logits[0].topk(4).indices
    tokens, last, length = ex.decode(m, first, 150, (Kp, Vp, plen), 4, 20, 30, 10)
    assert (length == 20).all()
    fed = torch.cat([first[None], tokens[:-1]])
    want0, want = _plain(m, prompt, first, fed)
    assert (logits[0].float() - want0.float()).abs().max() < 0.125
    assert (last.float() - want.float()).abs().max() < 0.125
    assert last.float().std() > 0.5


def test_evictions_bound_the_caches(ex):
    m = ex.ToyModel()
    prompt = torch.randint(0, 512, (300,), generator=torch.Generator().manual_seed(4)).cuda()
    logits, Kp, Vp, plen = ex.run_prompt(m, prompt, 100)
    assert (plen == 100).all()
    first = logits[0].topk(5).indices
    a = ex.decode(m, first, 300, (Kp, Vp, plen), 5, 100, 32, 16)
    b = ex.decode(m, first, 300, (Kp, Vp, plen), 5, 100, 32, 16)
    assert (a[2] == 32 + (100 - 48) % 16 + (16 if (100 - 48) % 16 == 0 else 0)).all()
    assert a[1].isfinite().all() and all(torch.equal(x, y) for x, y in zip(a, b))


def test_command_line(ex, capsys):
    ex.main("--samples 3 --prompt 200 --prefix-budget 64 --budget 32 --period 8 --tokens 50".split())
    assert "shared prefix of 64 rows" in capsys.readouterr().out
