"""Block-by-block decoding of a small masked-diffusion model over a 4-bit prefix cache.

The model (a few transformer layers with random weights, grouped heads, per-head norm and rotary
positions) decodes a block of masked positions at a time.  Its projections are torch's; what is
between them is this library's:

  fdllm_qk_norm_rope       queries and keys of the packed projection, normed and rotated
  fdllm_cache_attention    the block's queries over the cached prefix and the block's own keys
  fdllm_lmhead_select      which positions of the block to commit, and to what
  fdllm_cache_append       a finished block's keys and values into the 4-bit cache
  fdllm_cache_key_weights  the attention that each cached key received from the block
  fdllm_cache_evict        the cache brought down to the keys that received most

    python examples/cached_block_decoding.py [--batch 4] [--generate 128] [--budget 160]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_02955_gb300 as fd  # noqa: E402

EPS = 1e-6


def rms(x):
    """x over its root mean square, in fp32."""
    y = x.float()
    return (y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)).to(x.dtype)


class Model:
    """Random weights; the last token stands for a masked position."""

    def __init__(self, layers=2, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=1024, seed=0):
        g = torch.Generator().manual_seed(seed)

        def w(*shape):
            return (torch.randn(shape, generator=g) * shape[-1] ** -0.5).bfloat16().cuda()

        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed = (torch.randn(vocab, hidden, generator=g)).bfloat16().cuda()
        self.layers = [{"qkv": w((heads + 2 * kv_heads) * head_dim, hidden),
                        "out": w(hidden, heads * head_dim), "up": w(4 * hidden, hidden),
                        "down": w(hidden, 4 * hidden),
                        "q_norm": 1 + 0.1 * w(head_dim), "k_norm": 1 + 0.1 * w(head_dim)}
                       for _ in range(layers)]
        self.vocab_w = (8 * torch.randn(vocab, hidden, generator=g) * hidden ** -0.5).bfloat16().cuda()
        self.mask_token = vocab - 1
        self.inv_freq = 10000.0 ** (-torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2))


class PrefixCache:
    """A model's cached prefix: for each layer a 4-bit cache of pages and the weights its keys
    have received; two sets of pages a sequence, of which eviction fills the one not in use."""

    def __init__(self, model, batch, slots, page=32):
        per = -(-slots // page)
        self.caches = [fd.KvCache.empty(2 * batch * per, model.kv_heads, page, model.head_dim)
                       for _ in model.layers]
        pages = torch.randperm(2 * batch * per, generator=torch.Generator().manual_seed(1))
        self.table, self.other = pages.int().cuda().view(2, batch, per).contiguous()
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.longest = 0  # the host's bound of lens
        self.weights = [torch.zeros(batch, model.kv_heads, per * page, device="cuda")
                        for _ in model.layers]

    def append(self, state):
        """A block's keys and values behind what is there."""
        for cache, s in zip(self.caches, state):
            fd.fdllm_cache_append(cache, self.table, self.lens, s["k"], s["v"])
        self.lens = self.lens + state[0]["k"].shape[1]
        self.longest += state[0]["k"].shape[1]

    def count(self, state):
        """Adds what the cached keys received from a block's queries."""
        for cache, w, s in zip(self.caches, self.weights, state):
            fd.fdllm_cache_key_weights(s["q"], s["lse"], cache, self.table, self.lens, weights=w, out=w)

    def evict(self, budget, first, last):
        """Down to `budget` keys a sequence and head, if there are more."""
        if self.longest <= budget:
            return
        for i, cache in enumerate(self.caches):
            lens, kept, _ = fd.fdllm_cache_evict(cache, self.table, self.lens, self.weights[i], budget,
                                                 self.other, keep_first=first, keep_last=last)
            self.weights[i].zero_()
            self.weights[i][:, :, :budget] = kept
        self.lens, self.longest = lens, budget
        self.table, self.other = self.other, self.table


def forward(model, prefix, tokens, first):
    """Hidden states [B, n, H] of a block at positions first .. first + n - 1 and, of each layer,
    its queries, keys, values and attention's log-sum-exp."""
    B, n = tokens.shape
    at = torch.arange(first, first + n, dtype=torch.int32, device="cuda").repeat(B)
    x, state = model.embed[tokens.long()], []
    for layer, cache in zip(model.layers, prefix.caches):
        qkv = (rms(x) @ layer["qkv"].t()).view(B * n, -1, model.head_dim)
        q, k = fd.fdllm_qk_norm_rope(qkv[:, :model.heads], qkv[:, model.heads:-model.kv_heads], at,
                                     model.inv_freq, q_weight=layer["q_norm"],
                                     k_weight=layer["k_norm"], eps=EPS)
        q, k, v = (t.unflatten(0, (B, n)) for t in (q, k, qkv[:, -model.kv_heads:]))
        out, lse = fd.fdllm_cache_attention(q, cache, prefix.table, prefix.lens, k, v, return_lse=True)
        state.append({"q": q, "k": k, "v": v, "lse": lse})
        x = x + out.flatten(2) @ layer["out"].t()
        x = x + torch.nn.functional.silu(rms(x) @ layer["up"].t()) @ layer["down"].t()
    return rms(x), state


def decode(model, prompt, generate, block=32, budget=160, first=4, delta=0.25):
    """Tokens [B, generate] after prompt [B, P], the steps taken, and the cache."""
    B, P = prompt.shape
    prefix = PrefixCache(model, B, max(P, budget) + block)
    _, state = forward(model, prefix, prompt, 0)
    prefix.append(state)
    prefix.evict(budget, first, block)
    done, steps = [], 0
    for start in range(P, P + generate, block):
        n = min(block, P + generate - start)
        tokens = torch.full((B, n), model.mask_token, dtype=torch.int32, device="cuda")
        mask = torch.ones(B, n, dtype=torch.uint8, device="cuda")
        while bool(mask.any()):
            hidden, _ = forward(model, prefix, tokens, start)
            found, commit, _ = fd.fdllm_lmhead_select(hidden, model.vocab_w, mask, 1.0 - delta)
            tokens = torch.where(commit.bool(), found, tokens)
            steps += 1
        # the finished block: its own keys and values, and what it looked at
        _, state = forward(model, prefix, tokens, start)
        prefix.count(state)
        prefix.append(state)
        prefix.evict(budget, first, block)
        done.append(tokens)
    if fd.fdllm_cache_status() != 0:
        raise RuntimeError("a cache kernel reported an error")
    return torch.cat(done, 1), steps, prefix


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--generate", type=int, default=128)
    p.add_argument("--block", type=int, default=32)
    p.add_argument("--budget", type=int, default=160)
    a = p.parse_args()
    model = Model()
    g = torch.Generator().manual_seed(2)
    prompt = torch.randint(0, model.mask_token, (a.batch, a.prompt), generator=g).int().cuda()
    tokens, steps, prefix = decode(model, prompt, a.generate, a.block, a.budget)
    print("%d x %d tokens in %d steps; %s cached keys a sequence" %
          (a.batch, a.generate, steps, prefix.lens.tolist()))
    print(tokens[0, :16].tolist())


if __name__ == "__main__":
    main()
