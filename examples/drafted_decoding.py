"""Decoding with drafted tokens over a 4-bit prefix cache, the drafter trained as it goes.

A drafter (the next token's logits from the last token alone) proposes a chain of tokens drawn from
its own distribution, or a tree of its best ones; the target (the transformer of
cached_block_decoding.py) runs all of them in one pass, and what it takes is distributed as its own
samples.  What is between the projections is this library's:

  fdllm_qk_norm_rope          queries and keys, at the root's position plus the node's depth
  fdllm_tree_mask             which node sees which, and how deep it is
  fdllm_cache_tree_attention  the nodes' queries over the cached prefix and their ancestors' keys
  fdllm_verify_draft          the tokens taken, and the one that follows
  fdllm_cache_append          the taken nodes' keys and values into the 4-bit cache
  fdllm_distill_step          the drafter's loss on the target's top logits, and its gradient

    python examples/drafted_decoding.py [--batch 4] [--generate 64] [--tree]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from cached_block_decoding import EPS, Model, PrefixCache, fd, rms  # noqa: E402


class Drafter:
    """Logits of the next token from the last one: an embedding and a projection of its own."""

    rate = 0.1

    def __init__(self, vocab, hidden=128, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.embed = torch.randn(vocab, hidden, generator=g).bfloat16().cuda()
        self.head = (0.3 * torch.randn(vocab, hidden, generator=g) * hidden ** -0.5).cuda()

    def logits(self, tokens):
        return rms(self.embed[tokens.long()]) @ self.head.bfloat16().t()

    def learn(self, tokens, mask, target, top=32):
        """One step on the target's `top` logits and the rest of its mass, at the masked nodes."""
        x = rms(self.embed[tokens.long()])
        values, index = target.float().topk(top, -1)
        count = mask.sum().clamp(min=1)
        weights = (1.0 / count).expand(mask.shape).float().contiguous()
        loss, grad = fd.fdllm_distill_step((x @ self.head.bfloat16().t()), mask, index.int(), values,
                                           weights, teacher_lse=torch.logsumexp(target.float(), -1))
        self.head -= self.rate * (grad.flatten(0, 1).t() @ x.flatten(0, 1)).float()
        return loss.sum() / count


def draft_chain(drafter, root, nodes, g):
    """(tokens [B, nodes], the logits that each but the root was drawn from)."""
    tokens, rows = [root], []
    for _ in range(nodes - 1):
        rows.append(drafter.logits(tokens[-1]))
        race = torch.empty(rows[-1].shape, device="cuda").exponential_(generator=g)
        tokens.append((rows[-1].float() - race.log()).argmax(-1).int())
    return torch.stack(tokens, 1), torch.stack(rows, 1)


def draft_tree(drafter, root, parents):
    """Tokens [B, nodes] of a tree: the children of a node take the drafter's best after it."""
    tokens, used = [root], {}
    for p in parents[1:]:
        best = drafter.logits(tokens[p]).topk(used.get(p, 0) + 1, -1)[1]
        tokens.append(best[:, used.get(p, 0)].int())
        used[p] = used.get(p, 0) + 1
    return torch.stack(tokens, 1)


def forward_nodes(model, prefix, tokens, parents):
    """The target's logits [B, M, V] after each node of a tree, and each layer's keys and values."""
    B, M = tokens.shape
    mask, depth = fd.fdllm_tree_mask(parents)
    at = (prefix.lens[:, None] + depth).flatten().int()
    x, state = model.embed[tokens.long()], []
    for layer, cache in zip(model.layers, prefix.caches):
        qkv = (rms(x) @ layer["qkv"].t()).view(B * M, -1, model.head_dim)
        q, k = fd.fdllm_qk_norm_rope(qkv[:, :model.heads], qkv[:, model.heads:-model.kv_heads], at,
                                     model.inv_freq, q_weight=layer["q_norm"],
                                     k_weight=layer["k_norm"], eps=EPS)
        q, k, v = (t.unflatten(0, (B, M)) for t in (q, k, qkv[:, -model.kv_heads:]))
        out = fd.fdllm_cache_tree_attention(q, cache, prefix.table, prefix.lens, k, v, mask)
        state.append({"k": k, "v": v})
        x = x + out.flatten(2) @ layer["out"].t()
        x = x + torch.nn.functional.silu(rms(x) @ layer["up"].t()) @ layer["down"].t()
    return rms(x) @ model.vocab_w.t(), state


def step(model, drafter, prefix, root, nodes, tree, g, temperature=1.0, live=None):
    """One pass: draft, run, take, keep.  `tree`: the nodes' parents, or None for a chain; `live` [B]:
    the sequences that go on (None: all), the others keep their cache and teach nothing.  Returns
    what was taken and what it was made of."""
    B = root.shape[0]
    if tree is None:
        tokens, drawn = draft_chain(drafter, root, nodes, g)
        parents = torch.arange(-1, nodes - 1, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    else:
        tokens, drawn = draft_tree(drafter, root, tree), None
        parents = torch.tensor(tree, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    logits, state = forward_nodes(model, prefix, tokens, parents)
    uniform = torch.rand(tokens.shape, generator=g, device="cuda")
    noise = torch.empty((B, logits.shape[-1]), device="cuda").exponential_(generator=g)
    found, path, n = fd.fdllm_verify_draft(logits, tokens, parents=None if tree is None else parents,
                                           draft=drawn, temperature=temperature, uniform=uniform,
                                           noise=noise, draft_temperature=1.0)
    kept = n + 1 if live is None else torch.where(live, n + 1, 0)
    rows = path.clamp(min=0).long()[:, :, None, None].expand(-1, -1, model.kv_heads, model.head_dim)
    for cache, s in zip(prefix.caches, state):
        fd.fdllm_cache_append(cache, prefix.table, prefix.lens, s["k"].gather(1, rows),
                              s["v"].gather(1, rows), count=kept)
    on_path = torch.zeros(tokens.shape, dtype=torch.uint8, device="cuda")
    on_path.scatter_(1, path.clamp(min=0).long(), 1)
    if live is not None:
        on_path *= live[:, None]
    loss = drafter.learn(tokens, on_path, logits)
    before, prefix.lens = prefix.lens, prefix.lens + kept
    return {"tokens": found, "path": path, "n": n, "loss": loss, "nodes": tokens, "parents": parents,
            "logits": logits, "drawn": drawn, "uniform": uniform, "noise": noise, "state": state,
            "lens": before}


def decode(model, drafter, prompt, generate, nodes=6, tree=None, seed=0):
    """At least `generate` tokens of each sequence after prompt [B, P], the passes, and the losses."""
    B, P = prompt.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    nodes = nodes if tree is None else len(tree)
    prefix = PrefixCache(model, B, P + generate + nodes)
    chain = torch.arange(-1, P - 2, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    _, state = forward_nodes(model, prefix, prompt[:, :-1], chain)
    prefix.append(state)
    root, done, losses = prompt[:, -1], [[] for _ in range(B)], []
    while min(len(d) for d in done) < generate:
        # sequences that are done wait for the others
        live = torch.tensor([len(d) < generate for d in done], device="cuda")
        s = step(model, drafter, prefix, root, nodes, tree, g, live=live)
        root = torch.where(live, s["tokens"].gather(1, s["n"].clamp(min=0).long()[:, None])[:, 0], root)
        for d, row, n in zip(done, s["tokens"].tolist(), s["n"].tolist()):
            if len(d) >= generate:
                continue
            if n < 0:
                raise RuntimeError("a row of logits is not finite")
            d.extend(row[:n + 1])
        losses.append(float(s["loss"]))
    if fd.fdllm_cache_status() != 0:
        raise RuntimeError("a kernel reported an error")
    return done, losses, prefix


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--prompt", type=int, default=100)
    p.add_argument("--generate", type=int, default=64)
    p.add_argument("--tree", action="store_true")
    a = p.parse_args()
    model, drafter = Model(), Drafter(1024)
    prompt = torch.randint(0, model.mask_token, (a.batch, a.prompt), generator=torch.Generator().manual_seed(2))
    tree = [-1, 0, 0, 0, 1, 1, 2, 4] if a.tree else None
    done, losses, _ = decode(model, drafter, prompt.int().cuda(), a.generate, tree=tree)
    print("%s tokens in %d passes; the drafter's loss from %.2f to %.2f"
          % ([len(d) for d in done], len(losses), losses[0], losses[-1]))
    print(done[0][:16])


if __name__ == "__main__":
    main()
