"""Cases that measure drafting and its verification.

A drafter (a masked-diffusion model's block, or a smaller model) proposes a chain or a tree of
tokens, and a target model takes or rejects them.  The operators: the verification of the drafted
tokens from given random numbers (``verify``), the attention of a tree of drafted tokens over the
4-bit prefix cache and the tree's own keys (``tree``), and the loss that trains a drafter on its
target's top logits at the masked positions: forward (``loss``), loss and gradient in one call
(``step``), forward and backward through autograd (``back``).

Nodes of a draft: node 0 is the root, the last committed token; parents[b][j] < j.  Row j of
``target`` holds the target's logits after node j; row j of ``draft`` those that node j + 1 of a
chain was drawn from.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------- the cases
# `expect` of a verification: about how many rows of a sequence, from the root on, its path takes
# (its accepted nodes and the root); rows behind the first rejection need not be read.

def listed():
    return [
        # one sequence, four drafted tokens with the drafter's logits: latency
        {"name": "verify_chain_b1", "op": "verify", "B": 1, "M": 5, "V": 32000, "dtype": "bf16",
         "kind": "draft", "temperature": 1.0, "expect": 3.3},
        # a serving batch: chains of eight of different lengths over the diffusion model's vocabulary
        {"name": "verify_chain_b64", "op": "verify", "B": 64, "M": 9, "V": 126464, "dtype": "bf16",
         "kind": "draft", "temperature": 0.8, "expect": 3.1, "ragged": True},
        # trees of 48 nodes with the drafter's best tokens
        {"name": "verify_tree_b8", "op": "verify", "B": 8, "M": 48, "V": 126464, "dtype": "fp16",
         "kind": "tree", "temperature": 1.0, "expect": 1.7},
        # greedy verification of long chains, logits in 32 bits, a vocabulary of odd size
        {"name": "verify_greedy_odd", "op": "verify", "B": 16, "M": 17, "V": 50021, "dtype": "fp32",
         "kind": "greedy", "temperature": 0.0, "expect": 4.2},
        # one node a sequence: the next token alone; latency
        {"name": "tree_one_b1", "op": "tree", "B": 1, "M": 1, "Hq": 32, "Hk": 8, "D": 128,
         "dtype": "bf16", "page": 64, "low": 1021, "high": 1021},
        # the serving batch's trees over prefixes of different lengths, grouped heads
        {"name": "tree_serving_b32", "op": "tree", "B": 32, "M": 48, "Hq": 32, "Hk": 8, "D": 128,
         "dtype": "bf16", "page": 64, "low": 200, "high": 4096, "ragged": True, "empty": True},
        # wide trees over long prefixes, 64 channels, half precision
        {"name": "tree_long_d64", "op": "tree", "B": 2, "M": 255, "Hq": 16, "Hk": 16, "D": 64,
         "dtype": "fp16", "page": 128, "low": 30001, "high": 32000},
        # the loss on one block of one sequence, sixteen of the teacher's logits: latency
        {"name": "loss_block_b1", "op": "loss", "B": 1, "L": 32, "V": 126464, "K": 16,
         "dtype": "bf16", "temperature": 1.0, "rest": False, "masked": 1.0},
        # evaluation of a batch, logits in 32 bits, a vocabulary of odd size, the rest as one class
        {"name": "loss_eval_odd", "op": "loss", "B": 8, "L": 257, "V": 50021, "K": 100,
         "dtype": "fp32", "temperature": 2.0, "rest": True, "masked": 0.6},
        # a training step of one block of each of four sequences
        {"name": "step_block_b4", "op": "step", "B": 4, "L": 32, "V": 32000, "K": 32,
         "dtype": "bf16", "temperature": 1.0, "rest": False, "masked": 0.5},
        # a training step of a batch of sequences over the diffusion model's vocabulary
        {"name": "step_batch_b8", "op": "step", "B": 8, "L": 512, "V": 126464, "K": 64,
         "dtype": "bf16", "temperature": 1.0, "rest": True, "masked": 0.5},
        # the same loss inside a larger graph: forward, and backward from its gradient
        {"name": "back_b4", "op": "back", "B": 4, "L": 256, "V": 126464, "K": 64, "dtype": "fp16",
         "temperature": 1.5, "rest": False, "masked": 0.7},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["verify", "verify", "tree", "tree", "loss", "step", "back"])
    if op == "verify":
        c = {"op": op, "B": _log(rng, 1, 64), "M": _log(rng, 1, 64), "V": _log(rng, 50, 131072),
             "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
             "kind": rng.choice(["draft", "draft", "tree", "greedy"]), "ragged": rng.random() < 0.5}
        c["temperature"] = 0.0 if c["kind"] == "greedy" else rng.choice([0.5, 0.8, 1.0, 1.3])
        while c["B"] * c["M"] * c["V"] * (2 if c["dtype"] == "fp32" else 1) > 64 * 9 * 126464:
            c["B" if c["B"] > c["M"] else "M"] //= 2
        c["expect"] = min(3.0, float(c["M"]))
        return c
    if op == "tree":
        Hk, group = rng.choice([(32, 1), (8, 4), (16, 1), (4, 7), (2, 3)])
        c = {"op": op, "B": _log(rng, 1, 64), "M": _log(rng, 1, 257), "Hq": Hk * group, "Hk": Hk,
             "D": rng.choice([128, 128, 64]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
             "page": rng.choice([32, 64, 128, 256]), "ragged": rng.random() < 0.5,
             "empty": rng.random() < 0.3}
        high = _log(rng, 16, 32000)
        while c["B"] * high * Hk * c["D"] > 2 * 32000 * 16 * 64 or \
                c["B"] * (high + c["M"]) * c["Hq"] * c["M"] * c["D"] > 2 * 31000 * 16 * 255 * 64:
            if c["B"] > 1:
                c["B"] //= 2
            elif c["M"] > 64:
                c["M"] //= 2
            else:
                high //= 2
        c.update(high=high, low=int(high * rng.choice([0.1, 0.5, 1.0])))
        return c
    c = {"op": op, "B": _log(rng, 1, 16), "L": _log(rng, 1, 600), "V": _log(rng, 50, 131072),
         "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
         "temperature": rng.choice([0.7, 1.0, 2.0]), "rest": rng.random() < 0.5,
         "masked": rng.choice([0.15, 0.5, 1.0])}
    c["K"] = min(_log(rng, 1, 256), c["V"])
    while c["B"] * c["L"] * c["V"] * (2 if c["dtype"] == "fp32" else 1) > 8 * 300 * 126464:
        c["B" if c["B"] > 1 else "L"] //= 2
    return c


def _lens(c):
    """The cached lengths of a case's sequences, spread from `high` down to `low`; the last of a
    case with an empty sequence is 0."""
    lens = [c["high"] - int((c["high"] - c["low"]) * ((b * 0.6180339887) % 1.0)) for b in range(c["B"])]
    if c.get("empty") and c["B"] > 1:
        lens[-1] = 0
    return lens


def _nodes(c):
    """The counts of nodes of a case's drafts: every third is shorter in a ragged case."""
    return [c["M"] - (c["M"] // 3 if c.get("ragged") and b % 3 == 2 else 0) for b in range(c["B"])]


def _masked(c):
    rows = c["B"] * c["L"]
    return max(1, int(round(rows * c["masked"])))


def work(case):
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "verify":
        rows = c["B"] * min(c["expect"], c["M"])
        both = 2 if c["kind"] == "draft" and c["M"] > 1 else 1
        race = 0 if c["kind"] == "greedy" else 4 * c["B"] * c["V"]
        return {"bytes": rows * both * c["V"] * es + race, "flops": 4 * rows * both * c["V"]}
    if c["op"] == "tree":
        D, keys, nodes = c["D"], sum(_lens(c)), sum(_nodes(c))
        q = c["B"] * c["M"] * c["Hq"] * D * es
        # a node sees the cache and its ancestors: about the logarithm of the tree
        seen = sum(m * (n + math.log2(m + 1)) for n, m in zip(_lens(c), _nodes(c)))
        return {"bytes": 2 * q + 4 * c["B"] * c["M"] * c["Hq"] + keys * c["Hk"] * (D + 8) +
                2 * nodes * c["Hk"] * D * es + 12 * c["B"] * c["M"], "flops": 4 * c["Hq"] * D * seen}
    rows, all_rows, row = _masked(c), c["B"] * c["L"], c["V"] * es
    if c["op"] == "loss":
        return {"bytes": rows * (row + 8 * c["K"]) + 5 * all_rows, "flops": 4 * rows * c["V"]}
    return {"bytes": rows * (row + 8 * c["K"]) + all_rows * (row + 9), "flops": 8 * rows * c["V"]}


# ------------------------------------------------------------------------------- the inputs

def _logits(shape, g):
    """Logits as a head makes them: a Gaussian bulk and a few tokens well above it."""
    x = torch.randn(shape, generator=g, device="cuda").mul_(1.7)
    at = torch.randint(0, shape[-1], (*shape[:-1], 12), generator=g, device="cuda")
    up = 4.0 + 9.0 * torch.rand((*shape[:-1], 12), generator=g, device="cuda")
    return x.scatter_reduce_(-1, at, up, "amax")


def _keys_like(shape, g, tail):
    """Keys or values as a layer makes them: Gaussian, some channels several times larger, a mean."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.06
    x *= 1.0 + 2.0 * big.float()
    return x + tail * torch.randn(shape[-1], generator=g, device="cuda")


def _affine_codes(x):
    """Rows of D values in 32 bits -> (codes as numbers 0..15, scale, offset in bfloat16)."""
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale, offset = ((high - low) / 15.0).to(torch.bfloat16), low.to(torch.bfloat16)
    return ((x - offset.float()) / scale.float()).round_().clamp_(0, 15), scale, offset


def _pairs(codes):
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _trees(c, g):
    """Parents [B, M] of random trees (node 0: -1): a node hangs on one of the nodes before it,
    mostly on a near one, so that there are long paths and wide forks."""
    back = torch.rand((c["B"], c["M"]), generator=g, device="cuda") ** 3 * min(c["M"], 24)
    parents = torch.arange(c["M"], device="cuda") - 1 - back.long()
    parents = parents.clamp_(min=0)
    parents[:, 0] = -1
    return parents


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    return {"verify": _prepare_verify, "tree": _prepare_tree, "loss": _prepare_distill,
            "step": _prepare_distill, "back": _prepare_distill}[c["op"]](c, s, g)


def _prepare_verify(c, s, g):
    B, M, V, dt = c["B"], c["M"], c["V"], DTYPES[c["dtype"]]
    x = _logits((B, M, V), g)
    s["target"] = x.to(dt)
    s["lens"] = torch.tensor(_nodes(c), dtype=torch.int32, device="cuda")
    s["uniform"] = torch.rand((B, M), generator=g, device="cuda")
    noise = torch.empty((B, V), device="cuda").exponential_(generator=g)
    s["noise"] = noise.clamp_(min=1e-10)
    x = x + torch.randn(x.shape, generator=g, device="cuda") * (0.4 if c["kind"] == "greedy" else 0.6)
    tokens = torch.randint(0, V, (B, M), generator=g, device="cuda")
    if c["kind"] == "draft":
        # the drafter's logits, and tokens drawn from them at its own temperature
        s["draft"] = x[:, :M - 1].to(dt)
        race = torch.empty((B, M - 1, V), device="cuda").exponential_(generator=g).clamp_(min=1e-10)
        tokens[:, 1:] = (s["draft"].float() / c["temperature"] - race.log_()).argmax(-1)
    elif c["kind"] == "greedy":
        tokens[:, 1:] = x[:, :M - 1].argmax(-1)
    else:
        # a node's children carry the drafter's best tokens after it, best first
        parents = _trees(c, g)
        s["parents"] = parents.to(torch.int32)
        at = torch.arange(M, device="cuda")
        rank = ((parents[:, :, None] == parents[:, None]) & (at < at[:, None])).sum(-1)
        best = x.topk(min(32, V), -1)[1]
        up = best[torch.arange(B, device="cuda")[:, None], parents.clamp(min=0)]
        tokens[:, 1:] = up.gather(-1, (rank % best.shape[-1])[..., None])[:, 1:, 0]
    s["tokens"] = tokens.to(torch.int32)
    return s


def _prepare_tree(c, s, g):
    B, M, Hk, D, page, dt = c["B"], c["M"], c["Hk"], c["D"], c["page"], DTYPES[c["dtype"]]
    lens = _lens(c)
    per = max(1, -(-max(lens) // page))
    P = B * per + 3
    kc, ks, ko = _affine_codes(_keys_like((P, Hk, page, D), g, 0.3))
    s["k_codes"], s["k_affine"] = _pairs(kc), torch.cat((ks, ko), -1).contiguous()
    del kc
    vc, vs, vo = _affine_codes(_keys_like((P, Hk, page, D), g, 0.1))
    s["v_codes"] = _pairs(vc.transpose(-1, -2).contiguous())
    s["v_affine"] = torch.cat((vs, vo), -1).contiguous()
    table = torch.randperm(P, generator=g, device="cuda")[:B * per]
    s["table"] = table.to(torch.int32).view(B, per).contiguous()
    s["cache_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor(_nodes(c), dtype=torch.int32, device="cuda")
    s["parents"] = _trees(c, g).to(torch.int32)
    s["scale"] = D ** -0.5
    # rows of a packed projection: queries with some reach, so that the weights are not flat
    s["q"] = (1.5 * torch.randn((B, M, c["Hq"], D), generator=g, device="cuda")).to(dt)
    kv = torch.cat((_keys_like((B, M, Hk, D), g, 0.3), _keys_like((B, M, Hk, D), g, 0.1)), 2).to(dt)
    s["k_new"], s["v_new"] = kv[:, :, :Hk], kv[:, :, Hk:]
    return s


def _prepare_distill(c, s, g):
    B, L, V, K, T = c["B"], c["L"], c["V"], c["K"], c["temperature"]
    rows = B * L
    s["mask"] = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    s["mask"][torch.randperm(rows, generator=g, device="cuda")[:_masked(c)]] = 1
    s["mask"] = s["mask"].view(B, L)
    # distinct tokens, in the order of the teacher's logits; a few rows have fewer than K
    gap = torch.randint(1, V // K + 1, (B, L, K), generator=g, device="cuda").cumsum(-1) - 1
    index = gap.gather(-1, torch.rand((B, L, K), generator=g, device="cuda").argsort(-1))
    top = (14.0 - 6.0 * torch.rand((B, L, K), generator=g, device="cuda").cumsum(-1) / K ** 0.5)
    x = _logits((B, L, V), g)
    near = top + 1.0 * torch.randn((B, L, K), generator=g, device="cuda")
    s["logits"] = x.scatter_(-1, index, near).to(DTYPES[c["dtype"]])
    short = torch.rand((B, L, 1), generator=g, device="cuda") < 0.1
    gone = short & (torch.arange(K, device="cuda") >= max(1, K - K // 4))
    s["index"] = torch.where(gone, -1, index).to(torch.int32).contiguous()
    s["top"] = top.to(torch.bfloat16) if c["dtype"] == "bf16" else top
    s["lse"] = None
    if c["rest"]:
        # the rest of the teacher's vocabulary has 2 to 20 percent
        kept = (s["top"].float() / T).masked_fill(gone, -math.inf)
        rest = 0.02 + 0.18 * torch.rand((B, L), generator=g, device="cuda")
        s["lse"] = (torch.logsumexp(kept, -1) - torch.log1p(-rest)).contiguous()
    s["weights"] = torch.full((B, L), 1.0 / _masked(c), device="cuda")
    if c["dtype"] == "fp16":
        s["weights"] *= 8192.0  # the loss is scaled where gradients are in 16 bits of small range
    return s


# ------------------------------------------------------------------------------- the passes

def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _own_verify(s):
    import paper_2606_02955_gb300 as fd
    tokens, nodes, n = fd.fdllm_verify_draft(
        s["target"], s["tokens"], parents=s.get("parents"), lens=s["lens"], draft=s.get("draft"),
        temperature=s["case"]["temperature"], uniform=s["uniform"], noise=s["noise"])
    return {"tokens": tokens, "nodes": nodes, "n": n}


def _own_tree(s):
    import paper_2606_02955_gb300 as fd
    cache = fd.KvCache(s["k_codes"], s["v_codes"], s["k_affine"], s["v_affine"])
    mask, depth = fd.fdllm_tree_mask(s["parents"], s["lens"])
    out, lse = fd.fdllm_cache_tree_attention(s["q"], cache, s["table"], s["cache_lens"], s["k_new"],
                                             s["v_new"], mask, new_lens=s["lens"],
                                             scale=s["scale"], return_lse=True)
    return {"out": out, "lse": lse, "depth": depth}


def _own_loss(s):
    import paper_2606_02955_gb300 as fd
    return {"loss": fd.fdllm_distill_loss(s["logits"], s["mask"], s["index"], s["top"],
                                          teacher_lse=s["lse"],
                                          temperature=s["case"]["temperature"])}


def _own_step(s):
    import paper_2606_02955_gb300 as fd
    loss, grad = fd.fdllm_distill_step(s["logits"], s["mask"], s["index"], s["top"], s["weights"],
                                       teacher_lse=s["lse"], temperature=s["case"]["temperature"])
    return {"loss": loss, "grad": grad}


def _own_back(s):
    import paper_2606_02955_gb300 as fd
    x = s["logits"].detach().requires_grad_()
    loss = fd.fdllm_distill_loss(x, s["mask"], s["index"], s["top"], teacher_lse=s["lse"],
                                 temperature=s["case"]["temperature"])
    grad, = torch.autograd.grad(loss, x, s["weights"])
    return {"loss": loss.detach(), "grad": grad}


def _first_largest(x):
    """The lowest index of each row's largest value."""
    at = torch.arange(x.shape[-1], device="cuda")
    return torch.where(x == x.amax(-1, keepdim=True), at, x.shape[-1]).amin(-1)


def _softmax(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _above(parents, there):
    """Ancestors-or-self of each node: [B, M, M], true at (node, ancestor); the walk up doubles its
    length every turn."""
    M = parents.shape[1]
    at = torch.arange(M, device="cuda")
    up = (parents[..., None] == at) & (at < at[:, None]) | (at == at[:, None])
    up = (up & there[..., None] & there[:, None]).half()
    for _ in range(max(1, (M - 1).bit_length())):
        up = torch.matmul(up, up).clamp_(max=1.0)
    return up > 0


def _plain_verify(s):
    c = s["case"]
    B, M, V = c["B"], c["M"], c["V"]
    b, at = torch.arange(B, device="cuda"), torch.arange(M, device="cuda")
    lens, tokens = s["lens"].long()[:, None], s["tokens"].long()
    parents = s["parents"].long() if "parents" in s else (at - 1).expand(B, M)
    there = at < lens
    hung = there & (at > 0)
    over = parents.clamp(min=0)
    before = (parents[:, :, None] == parents[:, None]) & (at < at[:, None]) & hung[:, None] & hung[:, :, None]
    if c["kind"] == "greedy":
        best = _first_largest(s["target"])
        good = tokens == best.gather(1, over)
    else:
        p = _softmax(s["target"].float() / c["temperature"])
        here = p[b[:, None], over, tokens]
        u = s["uniform"].double()
        if c["kind"] == "draft":
            q = _softmax(s["draft"].float() / c["temperature"])
            drawn = torch.ones_like(here)
            drawn[:, 1:] = q.gather(-1, tokens[:, 1:, None])[..., 0]
            good = u * drawn.double() < here.double()
        else:
            again = (before & (tokens[:, :, None] == tokens[:, None])).any(-1)
            here = torch.where(again, 0.0, here).double()
            gone = (before * here[:, None]).sum(-1)
            good = u * (1.0 - gone) < here
    good = good & hung & ~(before & good[:, None]).any(-1)
    path = ~(_above(parents, there) & ~(good | (at == 0))[:, None]).any(-1) & there
    n = path.sum(-1) - 1
    nodes = torch.where(path, at, M).sort(-1)[0]
    last = nodes.gather(1, n[:, None])[:, 0]
    if c["kind"] == "greedy":
        extra = best[b, last]
    else:
        whole = p[b, last]
        if c["kind"] == "draft" and M > 1:
            less = q[b, last.clamp(max=M - 2)]
            left = torch.where((n + 1 < lens[:, 0])[:, None], (whole - less).clamp(min=0), whole)
        else:
            child = hung & (parents == last[:, None])
            left = torch.cat((whole, whole[:, :1]), 1)
            left = left.scatter(1, torch.where(child, tokens, V), 0.0)[:, :V]
        left = torch.where(left.amax(-1, keepdim=True) > 0, left, whole)
        extra = _first_largest(left / s["noise"])
    taken = tokens.gather(1, torch.cat((nodes[:, 1:], nodes[:, :1]), 1).clamp(max=M - 1))
    out = torch.where(at < n[:, None], taken, torch.where(at == n[:, None], extra[:, None], -1))
    nodes = torch.where(nodes < M, nodes, -1)
    return {"tokens": out.to(torch.int32), "nodes": nodes.to(torch.int32), "n": n.to(torch.int32)}


def _plain_tree(s):
    c = s["case"]
    B, M, Hq, Hk, D = c["B"], c["M"], c["Hq"], c["Hk"], c["D"]
    t = s["table"].long()

    def codes(x):
        return torch.stack((x & 15, x >> 4), -1).flatten(-2).float()

    def rows(x, affine, fresh):
        a = affine.float()
        x = (a[..., 1:2] + a[..., 0:1] * x).transpose(1, 2).flatten(2, 3)
        return torch.cat((x, fresh.float().transpose(1, 2)), 2)

    k = rows(codes(s["k_codes"][t]), s["k_affine"][t], s["k_new"])
    v = rows(codes(s["v_codes"][t]).transpose(-1, -2), s["v_affine"][t], s["v_new"])
    n = k.shape[2] - M
    node = torch.arange(M, device="cuda")
    above = _above(s["parents"].long(), node < s["lens"].long()[:, None])
    depth = torch.where(node < s["lens"][:, None], above.sum(-1) - 1, -1)
    seen = (torch.arange(n, device="cuda") < s["cache_lens"][:, None])[:, None].expand(B, M, n)
    seen = torch.cat((seen, above), 2).repeat(1, Hq // Hk, 1)[:, None]
    q = s["q"].float().view(B, M, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    x = (torch.matmul(q, k.transpose(-1, -2)) * s["scale"]).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(B, Hk, Hq // Hk, M, D).permute(0, 3, 1, 2, 4).reshape(B, M, Hq, D)
    lse = (top + torch.log(total)).view(B, Hk, Hq // Hk, M).permute(0, 3, 1, 2).reshape(B, M, Hq)
    return {"out": out.to(s["q"].dtype), "lse": lse, "depth": depth.to(torch.int32)}


def _plain_distill(s, gradient):
    c = s["case"]
    T, V = c["temperature"], c["V"]
    at = s["mask"].bool()
    x = s["logits"][at].float() / T
    index = s["index"][at].long()
    there = index >= 0
    # absent entries go to a column behind the vocabulary
    index = torch.where(there, index, V)
    t = (s["top"][at].float() / T).masked_fill(~there, -math.inf)
    x = x - x.amax(-1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(-1, keepdim=True)
    log_q = torch.nn.functional.pad(x, (0, 1)).gather(1, index) - torch.log(total)
    if s["lse"] is None:
        p = _softmax(t)
        log_p = torch.log(p)
    else:
        log_p = t - s["lse"][at][:, None]
        p = torch.exp(log_p)
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(-1)
    mass = p.sum(-1, keepdim=True)
    others = mass
    if s["lse"] is not None:
        left = (1.0 - mass).clamp(min=0)
        rest = torch.nn.functional.pad(e, (0, 1)).scatter(1, index, 0.0)[:, :V].sum(-1, keepdim=True) / total
        some = (left > 0) & (rest > 0)
        loss = loss + torch.where(some, left * (torch.log(left) - torch.log(rest)), 0.0)[:, 0]
        mass = torch.where(some, mass + left, mass)
        others = torch.where(some, mass - left / rest, mass)
    out = torch.zeros_like(s["weights"])
    out[at] = loss
    if not gradient:
        return {"loss": out}
    scale = (s["weights"][at] / T)[:, None]
    q = e / total
    dx = torch.nn.functional.pad(q * others, (0, 1))
    dx = dx.scatter(1, index, torch.nn.functional.pad(q, (0, 1)).gather(1, index) * mass - p)[:, :V]
    grad = torch.zeros_like(s["logits"])
    grad[at] = (dx * scale).to(grad.dtype)
    return {"loss": out, "grad": grad}


_own = {"verify": _own_verify, "tree": _own_tree, "loss": _own_loss, "step": _own_step,
        "back": _own_back}
_plain = {"verify": _plain_verify, "tree": _plain_tree, "loss": lambda s: _plain_distill(s, False),
          "step": lambda s: _plain_distill(s, True), "back": lambda s: _plain_distill(s, True)}


# ------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    if case["op"] == "verify":
        return None
    s = prepare(case, seed)
    return _exact_tree(s) if case["op"] == "tree" else _exact_distill(s)


def _rows64(s, b, which):
    """Sequence b's cached rows [Hk, slots, D] in 64 bits, from the bytes."""
    pages = s["table"][b].long()
    codes, affine = s[which + "_codes"][pages].int(), s[which + "_affine"][pages].double()
    x = torch.empty((*affine.shape[:3], s["case"]["D"]), dtype=torch.float64, device="cuda")
    if which == "k":
        x[..., 0::2], x[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    else:
        x[:, :, 0::2] = (codes % 16).double().transpose(2, 3)
        x[:, :, 1::2] = (codes // 16).double().transpose(2, 3)
    x = x * affine[..., :1] + affine[..., 1:]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])


def _exact_tree(s):
    c = s["case"]
    group = c["Hq"] // c["Hk"]
    out = torch.zeros((c["B"], c["M"], c["Hq"], c["D"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["B"], c["M"], c["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n, m = int(s["cache_lens"][b]), int(s["lens"][b])
        parents = s["parents"][b].tolist()
        sees = torch.zeros((c["M"], c["M"]), dtype=torch.bool)
        for i in range(m):
            at = i
            while at >= 0:
                sees[i, at] = True
                at = parents[at]
        hidden = ~sees[:, :m].cuda()
        k = torch.cat((_rows64(s, b, "k")[:, :n], s["k_new"][b, :m].double().transpose(0, 1)), 1)
        v = torch.cat((_rows64(s, b, "v")[:, :n], s["v_new"][b, :m].double().transpose(0, 1)), 1)
        for h in range(c["Hq"]):
            x = s["q"][b, :, h].double() @ k[h // group].t() * s["scale"]
            x[:, n:][hidden] = -math.inf
            lse[b, :, h] = torch.logsumexp(x, 1)
            out[b, :, h] = torch.nan_to_num(torch.softmax(x, 1)) @ v[h // group]
    return {"out": out, "lse": lse, "depth": None}


def _exact_distill(s):
    c = s["case"]
    T, V = c["temperature"], c["V"]
    loss = torch.zeros((c["B"], c["L"]), dtype=torch.float64, device="cuda")
    grad = torch.zeros((c["B"], c["L"], V), dtype=torch.float64, device="cuda") if c["op"] != "loss" else None
    for b in range(c["B"]):
        rows = s["mask"][b].nonzero()[:, 0]
        if not len(rows):
            continue
        log_q = torch.log_softmax(s["logits"][b, rows].double() / T, -1)
        index = s["index"][b, rows].long()
        t = s["top"][b, rows].double() / T
        t[index < 0] = -math.inf
        if s["lse"] is None:
            p = torch.softmax(t, -1)
        else:
            p = torch.exp(t - s["lse"][b, rows].double()[:, None])
        # the teacher's probabilities over the vocabulary, and which of them are its own
        listed_ = torch.zeros((len(rows), V), dtype=torch.bool, device="cuda")
        whole = torch.zeros((len(rows), V), dtype=torch.float64, device="cuda")
        r = torch.arange(len(rows), device="cuda")[:, None].expand_as(index)[index >= 0]
        listed_[r, index[index >= 0]] = True
        whole[r, index[index >= 0]] = p[index >= 0]
        terms = torch.where(whole > 0, whole * (torch.log(whole) - log_q), 0.0)
        value = terms.sum(-1)
        q = torch.exp(log_q)
        dx = q * whole.sum(-1, keepdim=True) - whole
        if s["lse"] is not None:
            left = (1.0 - whole.sum(-1, keepdim=True)).clamp(min=0)
            rest = torch.where(listed_, 0.0, q).sum(-1, keepdim=True)
            some = (left > 0) & (rest > 0)
            value = value + torch.where(some, left * (torch.log(left) - torch.log(rest)), 0.0)[:, 0]
            dx = dx + torch.where(some, left * (q - torch.where(listed_, 0.0, q) / rest), 0.0)
        loss[b, rows] = value
        if grad is not None:
            grad[b, rows] = dx * (s["weights"][b, rows].double() / T)[:, None]
    return {"loss": loss} if grad is None else {"loss": loss, "grad": grad}
