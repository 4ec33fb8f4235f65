"""Cases that measure the 4-bit prefix cache of block decoding and the query/key step before it.

A masked-diffusion model that decodes block by block keeps the keys and values of the prefix and
lets the active block's queries attend to them at every step.  The operators: the per-head norm and
rotation of queries and keys (``qk``), writing keys and values to the 4-bit cache and reading them
back (``store``), attention of a block over the cache and its own dense keys (``attn``), the
attention weight each cached key has received (``weigh``), and eviction by it (``evict``).

Cache: pages of ``page`` slots, found through a block table [B, pages per sequence].
  k_codes  [pages, heads, page, D/2]  uint8, channel 2i in the low half of byte i
  v_codes  [pages, heads, D, page/2]  uint8, slot 2i in the low half of byte i
  k_affine, v_affine [pages, heads, page, 2] bfloat16: (scale, offset) of a row of D values,
  value = offset + scale * code, code in 0..15.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------- the cases

def listed():
    return [
        # one active block of one sequence before attention: 32 positions, a 4096-wide layer of
        # 32 heads, rows taken from the packed qkv projection; launch latency
        {"name": "qk_block_b1", "op": "qk", "T": 32, "Hq": 32, "Hk": 32, "D": 128, "dtype": "bf16",
         "axes": 1, "norm": True, "interleaved": False, "top": 1024},
        # a batch of image-and-text prompts: three position axes, grouped heads
        {"name": "qk_prompt_axes3", "op": "qk", "T": 16381, "Hq": 32, "Hk": 8, "D": 128,
         "dtype": "bf16", "axes": 3, "norm": True, "interleaved": False, "top": 32768},
        # one committed token for each sequence of a serving batch, at odd slots
        {"name": "store_token_b64", "op": "store", "B": 64, "n": 1, "Hk": 32, "D": 128,
         "dtype": "bf16", "page": 64, "start": 777},
        # prompts of a batch entering the cache
        {"name": "store_prompt_b8", "op": "store", "B": 8, "n": 1021, "Hk": 32, "D": 128,
         "dtype": "bf16", "page": 64, "start": 3},
        # a single token of one sequence, grouped heads, half precision; latency
        {"name": "attn_token_b1_gqa", "op": "attn", "B": 1, "Lq": 1, "Ln": 1, "Hq": 32, "Hk": 8,
         "D": 128, "dtype": "fp16", "page": 64, "low": 1021, "high": 1021, "causal": False},
        # the serving batch's step: blocks of 32 over prefixes of 200 to 1024, one of them empty
        {"name": "attn_block_b64", "op": "attn", "B": 64, "Lq": 32, "Ln": 32, "Hq": 32, "Hk": 32,
         "D": 128, "dtype": "bf16", "page": 64, "low": 200, "high": 1024, "causal": False,
         "empty": True},
        # blocks of 64 over long prefixes with grouped heads: the tensor cores' share is largest
        {"name": "attn_long_gqa", "op": "attn", "B": 2, "Lq": 64, "Ln": 64, "Hq": 32, "Hk": 8,
         "D": 128, "dtype": "bf16", "page": 128, "low": 30001, "high": 32000, "causal": False},
        # a piece of a prompt: causal among its own keys, after a short cached prefix, 64 channels
        {"name": "attn_prompt_causal", "op": "attn", "B": 4, "Lq": 257, "Ln": 257, "Hq": 16,
         "Hk": 16, "D": 64, "dtype": "bf16", "page": 32, "low": 0, "high": 300, "causal": True},
        # key weights after a block of each of eight sequences
        {"name": "weigh_block_b8", "op": "weigh", "B": 8, "Lq": 32, "Hq": 32, "Hk": 32, "D": 128,
         "dtype": "bf16", "page": 64, "low": 500, "high": 1024},
        # key weights over long prefixes, grouped heads
        {"name": "weigh_long_gqa", "op": "weigh", "B": 2, "Lq": 64, "Hq": 32, "Hk": 8, "D": 128,
         "dtype": "bf16", "page": 128, "low": 30001, "high": 32000},
        # eight sequences brought down from a thousand cached keys to half
        {"name": "evict_b8", "op": "evict", "B": 8, "Hk": 32, "D": 128, "dtype": "bf16", "page": 64,
         "low": 500, "high": 1024, "budget": 512, "first": 4, "last": 64},
        # long prefixes brought down to a quarter
        {"name": "evict_long", "op": "evict", "B": 2, "Hk": 8, "D": 128, "dtype": "bf16",
         "page": 128, "low": 30001, "high": 32000, "budget": 8001, "first": 4, "last": 256},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["qk", "store", "attn", "attn", "weigh", "evict"])
    Hk, group = rng.choice([(32, 1), (8, 4), (16, 1), (4, 7), (2, 3)])
    D = rng.choice([128, 128, 64])
    c = {"op": op, "D": D, "dtype": rng.choice(["bf16", "bf16", "fp16"])}
    if op == "qk":
        c.update(T=_log(rng, 1, 16384), Hq=Hk * group, Hk=Hk, D=rng.choice([128, 64, 96, 256]),
                 dtype=rng.choice(["bf16", "fp16", "fp32"]), axes=rng.choice([1, 2, 3]),
                 norm=rng.random() < 0.8, interleaved=rng.random() < 0.3,
                 top=_log(rng, 64, 131072))
        while c["T"] * (c["Hq"] + Hk) * c["D"] * (2 if c["dtype"] == "fp32" else 1) > 16381 * 40 * 128:
            c["T"] = max(1, c["T"] // 2)
        return c
    c.update(Hk=Hk, page=rng.choice([32, 64, 128, 256]))
    if op == "store":
        c.update(B=_log(rng, 1, 64), n=_log(rng, 1, 1021), start=rng.randrange(0, 1000),
                 dtype=rng.choice(["bf16", "fp16", "fp32"]))
        while c["B"] * c["n"] * Hk * D > 8 * 1021 * 32 * 64:
            c["n"] = max(1, c["n"] // 2)
            c["B"] = max(1, c["B"] // 2)
        return c
    high = _log(rng, 16, 32000)
    c.update(B=_log(rng, 1, 64), high=high, low=int(high * rng.choice([0.3, 0.8, 1.0])))
    Lq = _log(rng, 1, 257)
    while c["B"] * c["high"] * Hk * D > 64 * 600 * 32 * 128 or \
            c["B"] * (c["high"] + Lq) * Hk * group * Lq * D > 2 * 31000 * 32 * 64 * 128:
        if c["B"] > 1:
            c["B"] //= 2
        elif Lq > 64:
            Lq //= 2
        else:
            c["high"] //= 2
    c["low"] = min(c["low"], c["high"])
    if op == "evict":
        c.update(budget=max(1, int(c["high"] * rng.choice([0.1, 0.25, 0.5, 0.9]))),
                 first=rng.choice([0, 4]), last=rng.choice([0, 16, 64]))
        c["first"] = min(c["first"], c["budget"])
        c["last"] = min(c["last"], c["budget"] - c["first"])
        return c
    c.update(Lq=Lq, Hq=Hk * group)
    if op == "attn":
        c.update(Ln=Lq, causal=rng.random() < 0.3, empty=rng.random() < 0.3)
    return c


def _lens(c):
    """The cached lengths of a case's sequences: spread from `high` down to `low`; the last of a
    case with an empty sequence is 0."""
    lens = [c["high"] - int((c["high"] - c["low"]) * ((b * 0.6180339887) % 1.0)) for b in range(c["B"])]
    if c.get("empty") and c["B"] > 1:
        lens[-1] = 0
    return lens


def work(case):
    c = case
    D, es = c["D"], 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "qk":
        values = c["T"] * (c["Hq"] + c["Hk"]) * D
        return {"bytes": 2 * values * es + 4 * c["axes"] * c["T"], "flops": 8 * values}
    if c["op"] == "store":
        rows = c["B"] * c["n"] * c["Hk"]
        return {"bytes": rows * 2 * (2 * D * es + D + 8), "flops": rows * 2 * 8 * D}
    lens = _lens(c)
    keys = sum(lens)
    if c["op"] == "evict":
        kept = c["Hk"] * sum(min(n, c["budget"]) for n in lens)
        return {"bytes": 4 * keys * c["Hk"] + kept * (3 * (D + 8) + 2 * D * es + 8),
                "flops": kept * 4 * D + 8 * keys * c["Hk"]}
    q = c["B"] * c["Lq"] * c["Hq"] * D * es
    if c["op"] == "weigh":
        return {"bytes": q + 4 * c["B"] * c["Lq"] * c["Hq"] + keys * c["Hk"] * (D // 2 + 4 + 8),
                "flops": 2 * c["Lq"] * c["Hq"] * D * keys}
    fresh = c["Ln"] * (c["Ln"] + 1) / 2 / c["Ln"] if c["causal"] else c["Ln"]
    return {"bytes": 2 * q + 4 * c["B"] * c["Lq"] * c["Hq"] + keys * c["Hk"] * (D + 8) +
            2 * c["B"] * c["Ln"] * c["Hk"] * D * es,
            "flops": 4 * c["Lq"] * c["Hq"] * D * (keys + c["B"] * fresh)}


# ------------------------------------------------------------------------------- the inputs

def _affine_codes(x):
    """Rows of D values in 32 bits -> (codes as numbers 0..15, scale, offset in bfloat16)."""
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((high - low) / 15.0).to(torch.bfloat16)
    offset = low.to(torch.bfloat16)
    s = scale.float()
    codes = ((x - offset.float()) / torch.where(s == 0, torch.ones_like(s), s)).round().clamp(0, 15)
    return torch.where(s == 0, torch.zeros_like(codes), codes), scale, offset


def _values(codes, affine):
    """(codes [..., D], affine [..., 2]) -> the values that they stand for, in 32 bits."""
    a = affine.float()
    return a[..., 1:2] + a[..., 0:1] * codes


def _pairs(codes):
    """Pack the last axis two to a byte, the first in the low half."""
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _unpairs(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2).float()


def _keys_like(shape, g, tail):
    """Keys or values as a layer makes them: Gaussian, some channels several times larger, a mean."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.06
    x *= torch.where(big, 3.0 * torch.ones_like(big, dtype=torch.float32), torch.ones_like(big, dtype=torch.float32))
    return x + tail * torch.randn(shape[-1], generator=g, device="cuda")


def _cache(c, pages_per_seq, g):
    """A filled cache: every sequence owns pages_per_seq pages, dealt in random order."""
    B, page, Hk, D = c["B"], c["page"], c["Hk"], c["D"]
    P = B * pages_per_seq + 3
    kc, ks, ko = _affine_codes(_keys_like((P, Hk, page, D), g, 0.3))
    k_codes, k_affine = _pairs(kc), torch.cat((ks, ko), -1)
    del kc
    vc, vs, vo = _affine_codes(_keys_like((P, Hk, page, D), g, 0.1))
    v_codes, v_affine = _pairs(vc.transpose(-1, -2).contiguous()), torch.cat((vs, vo), -1)
    table = torch.randperm(P, generator=g, device="cuda")[:B * pages_per_seq]
    return {"k_codes": k_codes, "v_codes": v_codes, "k_affine": k_affine.contiguous(),
            "v_affine": v_affine.contiguous(),
            "table": table.to(torch.int32).view(B, pages_per_seq).contiguous()}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, D = DTYPES[c["dtype"]], c["D"]
    s = {"case": c}
    if c["op"] == "qk":
        T, Hq, Hk = c["T"], c["Hq"], c["Hk"]
        # queries, keys and values of a packed projection: the rows of q and k are strided
        qkv = _keys_like((T, (Hq + 2 * Hk), D), g, 0.2).to(dt)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        s["wq"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dt) if c["norm"] else None
        s["wk"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dt) if c["norm"] else None
        s["pos"] = torch.randint(0, c["top"], (c["axes"], T), generator=g, device="cuda", dtype=torch.int32)
        pairs = D // 2
        s["inv_freq"] = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
        s["sections"] = [pairs // c["axes"]] * (c["axes"] - 1)
        s["sections"].append(pairs - sum(s["sections"]))
        # the same two on the device, for the plain form
        s["freq"] = s["inv_freq"].cuda()
        s["axis"] = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(s["sections"])).cuda()
        return s
    B, Hk, page = c["B"], c["Hk"], c["page"]
    if c["op"] == "store":
        per = -(-(c["start"] + c["n"] + 7) // page) + 1
        s.update(_cache(c, per, g))
        s["start"] = torch.tensor([c["start"] + b % 7 for b in range(B)], dtype=torch.int32, device="cuda")
        s["k"] = _keys_like((B, c["n"], Hk, D), g, 0.3).to(dt)
        s["v"] = _keys_like((B, c["n"], Hk, D), g, 0.1).to(dt)
        return s
    lens = _lens(c)
    per = max(1, -(-max(lens) // page))
    s.update(_cache(c, per, g))
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["op"] == "evict":
        # accumulated weights: most keys have little, a few much, some exactly the same
        w = torch.rand((B, Hk, per * page), generator=g, device="cuda")
        s["weights"] = torch.floor(1024 * (w ** 6) * 8) / 256
        need = -(-c["budget"] // page)
        P = s["k_codes"].shape[0]
        # room for the kept keys behind the pages in use
        for name in ("k_codes", "v_codes", "k_affine", "v_affine"):
            s[name] = torch.cat((s[name], torch.zeros((B * need,) + tuple(s[name].shape[1:]),
                                                      dtype=s[name].dtype, device="cuda")))
        s["to"] = (P + torch.randperm(B * need, generator=g, device="cuda")).to(torch.int32).view(B, need).contiguous()
        return s
    s["scale"] = D ** -0.5
    # queries after the norm and rotation, with some reach so that the weights are not flat
    s["q"] = (1.5 * torch.randn((B, c["Lq"], c["Hq"], D), generator=g, device="cuda")).to(dt)
    if c["op"] == "weigh":
        s["lse"] = math.log(max(lens)) + 1.5 + torch.rand((B, c["Lq"], c["Hq"]), generator=g, device="cuda")
        s["weights"] = torch.rand((B, Hk, per * page), generator=g, device="cuda")
        return s
    s["k_new"] = _keys_like((B, c["Ln"], Hk, D), g, 0.3).to(dt)
    s["v_new"] = _keys_like((B, c["Ln"], Hk, D), g, 0.1).to(dt)
    # the sequences' own counts of new keys: ragged in every third sequence
    new = [c["Ln"] - (c["Ln"] // 3 if b % 3 == 2 else 0) for b in range(B)]
    s["new_lens"] = torch.tensor(new, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------- the passes

def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _handle(s):
    import paper_2606_02955_gb300 as fd
    return fd, fd.KvCache(s["k_codes"], s["v_codes"], s["k_affine"], s["v_affine"])


def _own_qk(s):
    import paper_2606_02955_gb300 as fd
    q, k = fd.fdllm_qk_norm_rope(s["q"], s["k"], s["pos"], s["inv_freq"], q_weight=s["wq"],
                                 k_weight=s["wk"], eps=1e-6, sections=s["sections"],
                                 interleaved=s["case"]["interleaved"])
    return {"q": q, "k": k}


def _own_store(s):
    fd, cache = _handle(s)
    fd.fdllm_cache_append(cache, s["table"], s["start"], s["k"], s["v"])
    k, v = fd.fdllm_cache_read(cache, s["table"], s["start"], s["case"]["n"], s["k"].dtype)
    return {"k": k, "v": v}


def _own_attn(s):
    fd, cache = _handle(s)
    out, lse = fd.fdllm_cache_attention(s["q"], cache, s["table"], s["lens"], s["k_new"], s["v_new"],
                                      new_lens=s["new_lens"], causal=s["case"]["causal"],
                                      scale=s["scale"], return_lse=True)
    return {"out": out, "lse": lse}


def _own_weigh(s):
    fd, cache = _handle(s)
    return {"weights": fd.fdllm_cache_key_weights(s["q"], s["lse"], cache, s["table"], s["lens"],
                                                weights=s["weights"], scale=s["scale"])}


def _own_evict(s):
    fd, cache = _handle(s)
    c = s["case"]
    lens, weights, index = fd.fdllm_cache_evict(cache, s["table"], s["lens"], s["weights"], c["budget"],
                                              s["to"], keep_first=c["first"], keep_last=c["last"])
    k, v = fd.fdllm_cache_read(cache, s["to"], None, c["budget"], DTYPES[c["dtype"]], count=lens)
    return {"lens": lens, "weights": weights, "index": index, "k": k, "v": v}


def _plain_qk(s):
    c = s["case"]
    # position times frequency has more digits than 32 bits hold: the angle alone is in 64
    angle = s["pos"].double()[s["axis"]].t() * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
        if c["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y.chunk(2, -1)
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return y.to(x.dtype)

    return {"q": turn(s["q"], s["wq"]), "k": turn(s["k"], s["wk"])}


def _plain_store(s):
    c = s["case"]
    slot = s["start"].long()[:, None] + torch.arange(c["n"], device="cuda")
    page, at = torch.gather(s["table"].long(), 1, slot // c["page"]), slot % c["page"]
    kc, ks, ko = _affine_codes(s["k"].float())
    vc, vs, vo = _affine_codes(s["v"].float())
    s["k_codes"][page, :, at] = _pairs(kc)
    s["k_affine"][page, :, at] = torch.cat((ks, ko), -1)
    s["v_affine"][page, :, at] = torch.cat((vs, vo), -1)
    # values lie two slots to a byte: the pages that are written are unpacked, and packed again
    first, lead = s["start"].long() // c["page"], s["start"].long() % c["page"]
    cols = (c["n"] - 1) // c["page"] + 2
    pages = torch.gather(s["table"].long(), 1, first[:, None] + torch.arange(cols, device="cuda"))
    old = s["v_codes"][pages]
    v = torch.stack((old & 15, old >> 4), -1).flatten(-2).permute(0, 1, 4, 2, 3).flatten(1, 2)
    b = torch.arange(c["B"], device="cuda")[:, None]
    place = lead[:, None] + torch.arange(c["n"], device="cuda")
    v[b, place] = vc.to(torch.uint8)
    s["v_codes"][pages] = _pairs(v.unflatten(1, (cols, c["page"])).permute(0, 1, 3, 4, 2).contiguous())
    k = _values(_unpairs(s["k_codes"][page, :, at]), s["k_affine"][page, :, at])
    w = _values(v[b, place].float(), s["v_affine"][page, :, at])
    return {"k": k.to(s["k"].dtype), "v": w.to(s["v"].dtype)}


def _dense(s, codes_only_k=False):
    """Cached keys (and values) of every sequence in 32 bits: [B, Hk, pages * page, D]."""
    t = s["table"].long()
    k = _values(_unpairs(s["k_codes"][t]), s["k_affine"][t]).transpose(1, 2).flatten(2, 3)
    if codes_only_k:
        return k
    v = _values(_unpairs(s["v_codes"][t]).transpose(-1, -2), s["v_affine"][t])
    return k, v.transpose(1, 2).flatten(2, 3)


def _plain_attn(s):
    c = s["case"]
    B, Lq, Ln, Hq, Hk, D = c["B"], c["Lq"], c["Ln"], c["Hq"], c["Hk"], c["D"]
    k, v = _dense(s)
    n = k.shape[2]
    k = torch.cat((k, s["k_new"].float().transpose(1, 2)), 2)
    v = torch.cat((v, s["v_new"].float().transpose(1, 2)), 2)
    q = s["q"].float().view(B, Lq, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    x = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    at = torch.arange(n + Ln, device="cuda")
    seen = torch.where(at < n, at < s["lens"][:, None], at - n < s["new_lens"][:, None])[:, None]
    if c["causal"]:
        row = torch.arange(Lq, device="cuda")[:, None]
        seen = seen & ((at < n) | (at - n <= row))
    seen = seen.expand(B, Lq, n + Ln).repeat(1, Hq // Hk, 1)[:, None]
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(B, Hk, Hq // Hk, Lq, D).permute(0, 3, 1, 2, 4).reshape(B, Lq, Hq, D)
    lse = (top + torch.log(total)).view(B, Hk, Hq // Hk, Lq).permute(0, 3, 1, 2).reshape(B, Lq, Hq)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_weigh(s):
    c = s["case"]
    B, Lq, Hq, Hk, D = c["B"], c["Lq"], c["Hq"], c["Hk"], c["D"]
    k = _dense(s, codes_only_k=True)
    q = s["q"].float().view(B, Lq, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    lse = s["lse"].view(B, Lq, Hk, Hq // Hk).permute(0, 2, 3, 1).reshape(B, Hk, -1, 1)
    p = torch.exp(torch.matmul(q, k.transpose(-1, -2)) * s["scale"] - lse).sum(2)
    seen = torch.arange(k.shape[2], device="cuda") < s["lens"][:, None, None]
    return {"weights": torch.where(seen, s["weights"] + p, torch.zeros_like(p))}


def _plain_evict(s):
    c = s["case"]
    n, budget = s["weights"].shape[2], c["budget"]
    at = torch.arange(n, device="cuda")
    lens = s["lens"][:, None, None]
    rank = torch.where((at < c["first"]) | (at >= lens - c["last"]), math.inf, s["weights"])
    rank = torch.where(at < lens, rank, -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :budget]
    if best.shape[2] < budget:
        best = torch.nn.functional.pad(best, (0, budget - best.shape[2]), value=n)
    kept = torch.minimum(s["lens"], torch.full_like(s["lens"], budget))
    there = torch.arange(budget, device="cuda") < kept[:, None, None]
    best = torch.where(there, best, n).sort(-1)[0]
    index = torch.where(there, best, torch.full_like(best, -1)).to(torch.int32)
    from_ = torch.where(there, best, torch.zeros_like(best))
    weights = torch.where(there, torch.gather(s["weights"], 2, from_), torch.zeros_like(s["weights"][:1, :1, :1]))
    k, v = _dense(s)
    pick = from_[..., None].expand(-1, -1, -1, c["D"])

    def rows(x):
        x = torch.where(there[..., None], torch.gather(x, 2, pick), torch.zeros_like(x[:1, :1, :1, :1]))
        return x.transpose(1, 2).to(DTYPES[c["dtype"]])

    return {"lens": kept, "weights": weights, "index": index, "k": rows(k), "v": rows(v)}


_own = {"qk": _own_qk, "store": _own_store, "attn": _own_attn, "weigh": _own_weigh, "evict": _own_evict}
_plain = {"qk": _plain_qk, "store": _plain_store, "attn": _plain_attn, "weigh": _plain_weigh,
          "evict": _plain_evict}


# ------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"qk": _exact_qk, "store": _exact_store, "attn": _exact_attn, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["op"]](s)


def _exact_qk(s):
    c = s["case"]
    half = c["D"] // 2
    place = [(2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half) for i in range(half)]
    first = torch.tensor([a for a, _ in place], device="cuda")
    second = torch.tensor([b for _, b in place], device="cuda")
    axis = [a for a, n in enumerate(s["sections"]) for _ in range(n)]
    angle = torch.stack([s["pos"][a].double() * float(f) for a, f in zip(axis, s["inv_freq"])], 1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    out = {}
    for name, x, w in (("q", s["q"], s["wq"]), ("k", s["k"], s["wk"])):
        y = x.double()
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / c["D"] + 1e-6).sqrt() * w.double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def _exact_store(s):
    out = {}
    for name in ("k", "v"):
        x = s[name].double()
        low, high = x.min(-1, keepdim=True)[0], x.max(-1, keepdim=True)[0]
        step, base = ((high - low) / 15).to(torch.bfloat16).double(), low.to(torch.bfloat16).double()
        code = torch.nan_to_num((x - base) / step, nan=0.0, posinf=0.0, neginf=0.0)
        out[name] = base + step * torch.round(code).clamp(0, 15)
    return out


def _rows64(s, b, which):
    """Sequence b's cached rows [Hk, slots, D] in 64 bits, channel by channel from the bytes."""
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


def _exact_attn(s):
    c = s["case"]
    group = c["Hq"] // c["Hk"]
    out = torch.zeros((c["B"], c["Lq"], c["Hq"], c["D"]), dtype=torch.float64, device="cuda")
    lse = torch.full((c["B"], c["Lq"], c["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n, m = int(s["lens"][b]), int(s["new_lens"][b])
        if n + m == 0:
            continue
        k = torch.cat((_rows64(s, b, "k")[:, :n], s["k_new"][b, :m].double().transpose(0, 1)), 1)
        v = torch.cat((_rows64(s, b, "v")[:, :n], s["v_new"][b, :m].double().transpose(0, 1)), 1)
        for h in range(c["Hq"]):
            x = s["q"][b, :, h].double() @ k[h // group].t() * s["scale"]
            if c["causal"]:
                late = torch.arange(m, device="cuda")[None] > torch.arange(c["Lq"], device="cuda")[:, None]
                x[:, n:][late] = -math.inf
            lse[b, :, h] = torch.logsumexp(x, 1)
            out[b, :, h] = torch.softmax(x, 1) @ v[h // group]
    return {"out": out, "lse": lse}


def _exact_weigh(s):
    c = s["case"]
    group = c["Hq"] // c["Hk"]
    out = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n = int(s["lens"][b])
        k = _rows64(s, b, "k")
        out[b, :, :n] = s["weights"][b, :, :n].double()
        for h in range(c["Hq"]):
            x = s["q"][b, :, h].double() @ k[h // group, :n].t() * s["scale"]
            out[b, h // group, :n] += torch.exp(x - s["lse"][b, :, h, None].double()).sum(0)
    return {"weights": out}


def _exact_evict(s):
    c = s["case"]
    B, Hk, budget = c["B"], c["Hk"], c["budget"]
    k = torch.zeros((B, budget, Hk, c["D"]), dtype=torch.float64, device="cuda")
    v, w = torch.zeros_like(k), torch.zeros((B, Hk, budget), dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(s["lens"][b])
        kb, vb = _rows64(s, b, "k"), _rows64(s, b, "v")
        heavy = s["weights"][b, :, :n].cpu().tolist()
        for h in range(Hk):
            kept = list(range(n))
            if n > budget:
                middle = sorted(range(c["first"], n - c["last"]), key=lambda j: (-heavy[h][j], j))
                middle = middle[:budget - c["first"] - c["last"]]
                kept = sorted(list(range(c["first"])) + middle + list(range(n - c["last"], n)))
            at = torch.tensor(kept, dtype=torch.long, device="cuda")
            k[b, :len(kept), h], v[b, :len(kept), h] = kb[h, at], vb[h, at]
            w[b, h, :len(kept)] = s["weights"][b, h, at].double()
    return {"lens": None, "weights": w, "index": None, "k": k, "v": v}
