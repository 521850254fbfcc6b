"""Sampling several answers to one prompt with bounded caches.

A toy decoder (random weights, attention only) that uses the attention and eviction operators the way
a serving loop does:

1. the prompt runs once: ``attend`` with all its tokens as queries, accumulating every key's attention
   weight, then one ``evict`` of all layers copies the heaviest rows of its caches into a smaller cache;
2. that cache is the shared prefix of all samples: every decode step is one ``attend_shared`` per layer
   over the prefix (read once for all samples) and each sample's own rows;
3. every ``period`` steps one in-place ``evict`` of all layers cuts the samples' own caches back to
   their budget.

The cache lengths stay on the device; the host only counts steps.

    python examples/decode_with_eviction.py --samples 16 --prompt 2048 --prefix-budget 1024 \
        --budget 256 --period 64 --tokens 512
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_04971_gb300 import bkv  # noqa: E402


class ToyModel:
    """n_layers of causal grouped-query attention with residuals, RMS norms and rotary positions."""

    def __init__(self, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=512, rope_theta=1e4, seed=0,
                 device="cuda"):
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        self.device, self.dim = device, n_q_heads * head_dim
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols, gain=1.0):
            return (gain / math.sqrt(cols) * torch.randn(rows, cols, generator=g, device=device)).bfloat16()

        self.embed = torch.randn(vocab, self.dim, generator=g, device=device).bfloat16()
        self.qkv = [weight((n_q_heads + 2 * n_kv_heads) * head_dim, self.dim, 1.5) for _ in range(n_layers)]
        self.out = [weight(self.dim, self.dim) for _ in range(n_layers)]
        self.head = weight(vocab, self.dim)
        self.freq = rope_theta ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float32) / head_dim)

    @staticmethod
    def norm(x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()

    def rotate(self, x, pos):
        """x [batch, heads, n, head_dim] at positions pos [n]: pairs (i, i + head_dim / 2)."""
        a = pos.float()[:, None] * self.freq
        c, s = a.cos(), a.sin()
        lo, hi = x.float().chunk(2, -1)
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).bfloat16()

    def project(self, layer, h, pos):
        """h [batch, n, dim] -> q [batch, n_q_heads, n, d], k and v [batch, n_kv_heads, n, d], q and k rotated."""
        b, n, _ = h.shape
        x = (self.norm(h) @ self.qkv[layer].T).view(b, n, -1, self.head_dim).transpose(1, 2)
        q, k, v = x.split([self.n_q_heads, self.n_kv_heads, self.n_kv_heads], 1)
        return self.rotate(q, pos), self.rotate(k, pos), v.contiguous()

    def finish(self, layer, h, o):
        """Adds the attention output o [batch, n_q_heads, n, d] to the residual stream."""
        b, _, n, _ = o.shape
        return h + o.transpose(1, 2).reshape(b, n, self.dim) @ self.out[layer].T

    def logits(self, h):
        return self.norm(h) @ self.head.T


def run_prompt(m, tokens, prefix_budget, keep_last=16, keep_first=4):
    """The prompt's pass.  Returns its last logits and the shared prefix: K, V [n_layers, 1, n_kv_heads,
    prefix_budget, d] and lengths int32 [n_layers, 1, n_kv_heads]."""
    n = tokens.numel()
    bk = bkv.BeaconKV(n_layers=m.n_layers, batch=1, n_q_heads=m.n_q_heads, n_kv_heads=m.n_kv_heads,
                      head_dim=m.head_dim, n_beacons=0, window=keep_last, n_prefix=keep_first, capacity=n)
    shape = (m.n_layers, 1, m.n_kv_heads)
    K = torch.empty(*shape, n, m.head_dim, dtype=torch.bfloat16, device=m.device)
    V = torch.empty_like(K)
    weights = torch.zeros(*shape, n, device=m.device)
    length = torch.full(shape, n, dtype=torch.int32, device=m.device)
    bk.reserve_attend(n_q=n, weights=True)
    pos = torch.arange(n, device=m.device)
    h = m.embed[tokens][None]
    for layer in range(m.n_layers):
        q, K[layer], V[layer] = m.project(layer, h, pos)
        o, _ = bk.attend(q, K[layer], V[layer], length=length[layer], weights=weights[layer])
        h = m.finish(layer, h, o)
    Kp = torch.zeros(*shape, prefix_budget, m.head_dim, dtype=torch.bfloat16, device=m.device)
    Vp, wp = torch.zeros_like(Kp), torch.empty(*shape, prefix_budget, device=m.device)
    _, prefix_len = bk.evict(K, V, weights, L=length, budget=prefix_budget, K_out=Kp, V_out=Vp, weights_out=wp)
    bk.sync()
    bk.close()
    return m.logits(h[:, -1]), Kp, Vp, prefix_len


def decode(m, first, prompt_len, prefix, samples, n_tokens, budget, period, keep_last=16):
    """n_tokens greedy steps of `samples` samples from the tokens `first` [samples].  Returns the tokens
    [n_tokens, samples], the logits of the last step and the own caches' lengths."""
    Kp, Vp, prefix_len = prefix
    cap = budget + period
    bk = bkv.BeaconKV(n_layers=m.n_layers, batch=samples, n_q_heads=m.n_q_heads, n_kv_heads=m.n_kv_heads,
                      head_dim=m.head_dim, n_beacons=0, window=keep_last, capacity=cap)
    shape = (m.n_layers, samples, m.n_kv_heads)
    K = torch.zeros(*shape, cap, m.head_dim, dtype=torch.bfloat16, device=m.device)
    V, weights = torch.zeros_like(K), torch.zeros(*shape, cap, device=m.device)
    length = torch.zeros(shape, dtype=torch.int32, device=m.device)
    kept = torch.empty(*shape, budget, dtype=torch.int32, device=m.device)
    prefix_rows = prefix_len[:, :, 0].contiguous()  # the same for all KV heads of a layer
    bk.reserve_attend(n_q=1, n_groups=1, weights=True)
    b = torch.arange(samples, device=m.device)[:, None]
    kv = torch.arange(m.n_kv_heads, device=m.device)[None]
    rows = 0  # of every own cache; the same number everywhere, so the host can count it
    tokens, logits, token = [], None, first
    for step in range(n_tokens):
        if rows == cap:
            bk.evict(K, V, weights, L=length, budget=budget, kept_out=kept, len_out=length)
            rows = budget
        pos = torch.tensor([prompt_len + step], device=m.device)
        h = m.embed[token][:, None]
        for layer in range(m.n_layers):
            q, k, v = m.project(layer, h, pos)
            at = length[layer].long()
            K[layer][b, kv, at], V[layer][b, kv, at] = k[:, :, 0], v[:, :, 0]
            length[layer] += 1
            o, _ = bk.attend_shared(q, Kp[layer], Vp[layer], K[layer], V[layer], prefix_len=prefix_rows[layer],
                                    length=length[layer], weights=weights[layer])
            h = m.finish(layer, h, o)
        rows += 1
        logits = m.logits(h[:, 0])
        token = logits.argmax(-1)
        tokens.append(token)
    bk.sync()
    bk.close()
    return torch.stack(tokens), logits, length


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--samples", type=int, default=16)
    p.add_argument("--prompt", type=int, default=2048, help="tokens of the prompt")
    p.add_argument("--prefix-budget", type=int, default=1024, help="rows of the prompt's caches that stay")
    p.add_argument("--budget", type=int, default=256, help="rows of a sample's own cache after an eviction")
    p.add_argument("--period", type=int, default=64, help="decode steps between two evictions")
    p.add_argument("--tokens", type=int, default=512)
    a = p.parse_args(argv)
    m = ToyModel()
    prompt = torch.randint(0, m.embed.shape[0], (a.prompt,), generator=torch.Generator().manual_seed(1)).cuda()
    logits, Kp, Vp, prefix_len = run_prompt(m, prompt, a.prefix_budget)
    first = logits[0].topk(a.samples).indices  # every sample starts with another token
    torch.cuda.synchronize()
    t = time.perf_counter()
    tokens, _, length = decode(m, first, a.prompt, (Kp, Vp, prefix_len), a.samples, a.tokens, a.budget, a.period)
    ms = (time.perf_counter() - t) * 1e3 / a.tokens
    print(f"prompt {a.prompt} tokens -> shared prefix of {int(prefix_len.max())} rows; {a.samples} samples x {a.tokens} "
          f"tokens, own caches at {int(length.min())}..{int(length.max())} rows, {ms:.2f} ms per step")
    print("first sample's tokens:", tokens[:12, 0].tolist())


if __name__ == "__main__":
    main()
