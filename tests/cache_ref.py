"""Plain 64-bit references of the 4-bit prefix cache's operators, and seeded inputs for them.

Written from the operators' formulas with loops over sequences and heads; nothing here is
shared with the library's code.  Tolerances used with them (fixed before the first run):

  * attention output: half an ulp of the output type (its unit roundoff: 2^-8 for bfloat16's 8
    significant bits, 2^-11 for fp16's 11); the weights' rounding to fp16 (2^-11) times what
    they multiply (codes: up to 15 scales of the row; own values: |v|); scores off by `d` change
    a weight by at most a factor e^(2 d).
    Scores are fp32 sums of products of queries with codes, up to 15 scales, and of the row's
    offset: d = 2^-21 * scale * max_j sum_c |q_c| (|offset_j| + 15 scale_j), which leaves the sum
    8 roundings of its largest partial sum (own keys: |k| in the bracket's place).
  * lse: d, and four fp32 roundings of the result.
  * key weights: the same 2 d on every term, and n fp32 roundings of the sum.
"""
import math

import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def quantise(x):
    """Rows [..., D] -> (codes 0..15 int64, scale, offset bfloat16), in fp32 as documented."""
    x = x.float().cpu()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((high - low) / torch.full_like(high, 15.0)).bfloat16()
    offset = low.bfloat16()
    bad = ~(torch.isfinite(scale.float()) & torch.isfinite(offset.float())) | \
        ~torch.isfinite(x).all(-1, keepdim=True)
    s = scale.float()
    safe = torch.where((s == 0) | bad, torch.ones_like(s), s)
    codes = torch.round((x - offset.float()) / safe).clamp(0, 15)
    codes = torch.where((s == 0) | bad, torch.zeros_like(codes), torch.nan_to_num(codes))
    nan = torch.full_like(scale, math.nan)
    return codes.long(), torch.where(bad, nan, scale), torch.where(bad, nan, offset)


def values(x):
    """The values that rows are held as, in fp64."""
    codes, scale, offset = quantise(x)
    return offset.double() + scale.double() * codes.double()


def unpack_cache(cache):
    """(k, v) [pages, heads, page, D] fp64 of a KvCache's tensors."""
    kc, vc = cache.k_codes.cpu().long(), cache.v_codes.cpu().long()
    k = torch.stack((kc & 15, kc >> 4), -1).flatten(-2).double()
    v = torch.stack((vc & 15, vc >> 4), -1).flatten(-2).transpose(-1, -2).double()
    ka, va = cache.k_affine.cpu().double(), cache.v_affine.cpu().double()
    return k * ka[..., :1] + ka[..., 1:], v * va[..., :1] + va[..., 1:]


def sequence(dense, table_row, page, n):
    """The first n cached rows of a sequence [heads, n, D]."""
    pages = table_row.cpu().long()[:-(-n // page)] if n else table_row.cpu().long()[:0]
    x = dense[pages].transpose(0, 1)
    return x.reshape(dense.shape[1], -1, dense.shape[3])[:, :n]


def row_reach(affine, D):
    """|offset| + 15 scale of every cached row, as [pages, heads, page, D]."""
    f = affine.cpu().double()
    return (f[..., 1:].abs() + 15 * f[..., :1]).expand(-1, -1, -1, D)


def attention(q, cache, table, lens, k_new=None, v_new=None, new_lens=None, causal=False,
              scale=None):
    """(out, lse, tolerance of out, tolerance of lse), fp64 on the CPU."""
    kd, vd = unpack_cache(cache)
    k_reach = row_reach(cache.k_affine, cache.head_dim)
    v_reach = (15 * cache.v_affine[..., :1].cpu().double()).expand(-1, -1, -1, cache.head_dim)
    q64 = q.cpu().double()
    B, Lq, Hq, D = q64.shape
    group = Hq // cache.heads
    scale = D ** -0.5 if scale is None else scale
    out = torch.zeros(B, Lq, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Lq, Hq), -math.inf, dtype=torch.float64)
    tol = torch.zeros_like(out)
    tol_lse = torch.zeros_like(lse)
    for b in range(B):
        n = int(lens[b])
        k, v, kr, vr = (sequence(x, table[b], cache.page_size, n) for x in (kd, vd, k_reach, v_reach))
        vr = torch.maximum(v.abs(), vr)
        m = 0
        if k_new is not None:
            m = k_new.shape[1] if new_lens is None else int(new_lens[b])
            own_k, own_v = (x[b, :m].cpu().double().transpose(0, 1) for x in (k_new, v_new))
            k, v = torch.cat((k, own_k), 1), torch.cat((v, own_v), 1)
            kr, vr = torch.cat((kr, own_k.abs()), 1), torch.cat((vr, own_v.abs()), 1)
        for h in range(Hq):
            kh, vh, krh, vrh = (x[h // group] for x in (k, v, kr, vr))
            for i in range(Lq):
                seen = n + (min(m, i + 1) if causal else m)
                if seen == 0:
                    continue
                x = kh[:seen] @ q64[b, i, h] * scale
                d = 2.0 ** -21 * abs(scale) * float((krh[:seen] @ q64[b, i, h].abs()).max())
                lse[b, i, h] = torch.logsumexp(x, 0)
                p = torch.softmax(x, 0)
                out[b, i, h] = p @ vh[:seen]
                spread = p @ vrh[:seen]
                tol[b, i, h] = EPS[q.dtype] * out[b, i, h].abs() + (2.0 ** -11 + 2 * d) * spread + 1e-30
                tol_lse[b, i, h] = d + 4 * 2.0 ** -24 * max(1.0, abs(float(lse[b, i, h]))) + 1e-6
    return out, lse, tol, tol_lse


def key_weights(q, lse, cache, table, lens, weights, scale=None):
    """(weights, tolerance) fp64 [B, heads, max_len]."""
    kd, _ = unpack_cache(cache)
    k_reach = row_reach(cache.k_affine, cache.head_dim)
    q64, lse64 = q.cpu().double(), lse.cpu().double()
    B, Lq, Hq, D = q64.shape
    group = Hq // cache.heads
    scale = D ** -0.5 if scale is None else scale
    w = torch.zeros_like(weights.cpu().double())
    tol = torch.zeros_like(w)
    for b in range(B):
        n = int(lens[b])
        k = sequence(kd, table[b], cache.page_size, n)
        kr = sequence(k_reach, table[b], cache.page_size, n)
        for h in range(cache.heads):
            qh = q64[b, :, h * group:(h + 1) * group].reshape(-1, D)
            ls = lse64[b, :, h * group:(h + 1) * group].reshape(-1, 1)
            p = torch.exp(qh @ k[h].t() * scale - ls)
            p = torch.where(torch.isinf(ls) & (ls < 0), torch.zeros_like(p), p)
            d = 2.0 ** -21 * abs(scale) * (qh.abs() @ kr[h].t())
            # exp's argument, in base 2: two roundings of it and of the exponential
            d = d + 2.0 ** -22 * (2 + torch.nan_to_num(ls, neginf=0.0).abs() + (qh @ k[h].t() * scale).abs())
            w[b, h, :n] = weights[b, h, :n].cpu().double() + p.sum(0)
            tol[b, h, :n] = (2 * d * p).sum(0) + 2.0 ** -24 * (p.shape[0] + 4) * w[b, h, :n].abs()
    return w, tol


def make_cache(fd, lens, heads, D, page, seed, spare=3, poison=True, min_pages=1):
    """A KvCache filled through its own tensors with quantised Gaussian rows, every sequence's
    pages dealt in random order; slots behind the lengths hold NaN scales when `poison`."""
    g = torch.Generator().manual_seed(seed)
    per = max(min_pages, max(-(-n // page) for n in lens))
    B = len(lens)
    pages = B * per + spare
    k = torch.randn(pages, heads, page, D, generator=g) * (1 + 2 * (torch.rand(D, generator=g) < 0.1)) + 0.2
    v = torch.randn(pages, heads, page, D, generator=g) + 0.1 * torch.randn(D, generator=g)
    table = torch.randperm(pages, generator=g)[:B * per].view(B, per).int()
    kc, ks, ko = quantise(k)
    vc, vs, vo = quantise(v)
    ka, va = torch.cat((ks, ko), -1), torch.cat((vs, vo), -1)
    if poison:
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(n):
                used[int(table[b, j // page]), j % page] = True
        ka[~used[:, None].expand(-1, heads, -1)] = math.nan
        va[~used[:, None].expand(-1, heads, -1)] = math.inf
    kp = (kc[..., 0::2] | (kc[..., 1::2] << 4)).to(torch.uint8)
    vt = vc.transpose(-1, -2)
    vp = (vt[..., 0::2] | (vt[..., 1::2] << 4)).to(torch.uint8)
    cache = fd.KvCache(kp.contiguous().cuda(), vp.contiguous().cuda(), ka.contiguous().cuda(),
                       va.contiguous().cuda())
    return cache, table.cuda()


def rope(x, weight, positions, sections, inv_freq, eps, interleaved):
    """fp64 per-head norm and rotation of x [T, H, D]."""
    y = x.cpu().double()
    T, H, D = y.shape
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.cpu().double()
    pos = positions.cpu().long().view(-1, T)
    pairs = len(inv_freq)
    axis = [a for a, n in enumerate(sections or [pairs]) for _ in range(n)]
    out = y.clone()
    for p in range(pairs):
        # position * frequency with the whole turns taken off in rational steps
        f = float(inv_freq[p])
        angle = torch.tensor([math.fmod(int(t) * f, 2 * math.pi) for t in pos[axis[p]]],
                             dtype=torch.float64)[:, None]
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
        c, s = torch.cos(angle), torch.sin(angle)
        out[..., i] = y[..., i] * c - y[..., j] * s
        out[..., j] = y[..., j] * c + y[..., i] * s
    return out
