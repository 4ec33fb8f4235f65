"""Plain 64-bit references of drafting's operators (verification, tree masks, distillation), with
loops over sequences and nodes; nothing here is shared with the library's code.

Tolerances of the distillation (fixed before the first run).  With u = 2^-24:
  * A sum of exponentials: each term is off by 2^-22 (ex2.approx) and by its argument's four
    roundings, |t| u ln 2 each (t in bits); a term weighs 2^-t, so the arguments take at most
    4 u ln 2 times the mean of t over the distribution, which its entropy and so log2 V bounds; and
    the additions take u for each of a thread's own (V / 256 of them) and 40 for the joins.
      z = 2^-22 + u (4 log2 V + V / 256 + 40)
  * The teacher's probabilities: exponent and division, 8 u, and the roundings of their arguments
    (t / temperature and the log-sum-exp, at most 64 here), 2 * 64 u; sums of up to 1024: 16 u.
      p = 8 u + 128 u + 16 u = 152 u
  * A loss of terms m (log a - log b): each mass off by p, each logarithm off by z + p and by the
    rounding of what it is made of, 4 u (|log a| + |x - M| / temperature + log Z).  The rest's mass
    R is 1 less a sum, off by p absolutely.
  * A gradient: the formula's terms off by 2 (z + p) each, and half a step of the result's type
    (2^-8, 2^-11, 2^-24; below the normal numbers half of the smallest subnormal).  Its q_v and
    q_v / r are single exponentials: the four roundings of an argument of t bits take 4 u ln 2 |t| of
    them, whatever they weigh in the sum; and the exponential is 0 below 2^-126 (ex2.approx.ftz), so
    2^-126 of the factor before it, |grad_loss| / temperature (P + 2 R), may be lost besides.
"""
import math

import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}
U = 2.0 ** -24


def tree_mask(parents, lens=None):
    """(sees bool [B, M, M], depth int64 [B, M])."""
    B, M = parents.shape
    sees = torch.zeros(B, M, M, dtype=torch.bool)
    depth = torch.full((B, M), -1, dtype=torch.int64)
    for b in range(B):
        n = M if lens is None else min(max(int(lens[b]), 0), M)
        for i in range(n):
            at, steps = i, 0
            sees[b, i, i] = True
            while at > 0 and 0 <= int(parents[b, at]) < at:
                at, steps = int(parents[b, at]), steps + 1
                sees[b, i, at] = True
            depth[b, i] = steps
    return sees, depth


def bits(sees):
    """bool [..., n] -> int32 [..., ceil(n / 32)], bit j % 32 of word j / 32."""
    n = sees.shape[-1]
    pad = torch.nn.functional.pad(sees.long(), (0, -n % 32)).unflatten(-1, (-1, 32))
    words = (pad << torch.arange(32)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def softmax64(row, temperature):
    """fp64 softmax of a row, or None where it holds a NaN or its maximum is infinite."""
    x = row.double()
    if torch.isnan(x).any() or not math.isfinite(float(x.max())):
        return None
    return torch.softmax(x / temperature, 0)


def verify(target, tokens, parents=None, lens=None, draft=None, temperature=1.0,
           draft_temperature=None, uniform=None, noise=None):
    """(tokens, nodes, n, margin): the margin is the smallest relative distance of a test or of a
    draw's two best tokens from equality, per sequence (inf where nothing could tip)."""
    target, tokens = target.cpu(), tokens.cpu()
    B, M, V = target.shape
    draft_temperature = temperature if draft_temperature is None else draft_temperature
    out = torch.full((B, M), -1, dtype=torch.int32)
    nodes = torch.full((B, M), -1, dtype=torch.int32)
    count = torch.zeros(B, dtype=torch.int32)
    margin = [math.inf] * B
    greedy = temperature == 0.0
    for b in range(B):
        n = M if lens is None else min(max(int(lens[b]), 1), M)
        up = [-1] + [j - 1 if parents is None else int(parents[b, j]) for j in range(1, M)]
        up = [p if 0 <= p < j else -1 for j, p in enumerate(up)]
        path, cur, bad, left, tried, rejected = [0], 0, False, 1.0, [], False

        def rows(c):
            p = softmax64(target[b, c], 1.0 if greedy else temperature)
            q = None
            if draft is not None and c < n - 1:
                q = softmax64(draft.cpu()[b, c], draft_temperature)
                if q is None:
                    return None, None
            return p, q

        def best(w):
            return int((w == w.max()).nonzero()[0, 0])

        p, q = rows(0)
        bad = p is None
        for j in range(1, n):
            if bad or rejected:
                break
            if up[j] != cur:
                continue
            d = int(tokens[b, j])
            inside = 0 <= d < V
            if greedy:
                ok = inside and d == best(target[b, cur].double())
            else:
                u = float(uniform[b, j])
                pd = float(p[d]) if inside and d not in tried else 0.0
                side = u * (float(q[d]) if inside else 0.0) if q is not None else u * left
                ok = side < pd
                if max(side, pd) > 0 and pd > 0:
                    margin[b] = min(margin[b], abs(side - pd) / max(side, pd))
            if ok:
                cur, left, tried = j, 1.0, []
                path.append(j)
                p, q = rows(cur)
                bad = p is None
            else:
                tried.append(d)
                left -= 0.0 if greedy else pd
                rejected = draft is not None
        if bad:
            count[b] = -1
            margin[b] = math.inf
            continue
        if greedy:
            extra = best(target[b, cur].double())
        else:
            r = p.clone()
            if rejected:
                r = (p - q).clamp(min=0)
            elif draft is None:
                for d in tried:
                    if 0 <= d < V:
                        r[d] = 0.0
            if float(r.max()) <= 0:
                r = p
            e = noise[b].cpu().double()
            key = torch.where((r > 0) & (e >= 0) & torch.isfinite(e), r / e, torch.zeros_like(r))
            two = key.topk(min(2, V))[0].tolist()
            if len(two) == 2 and two[0] > 0 and math.isfinite(two[0]):
                margin[b] = min(margin[b], (two[0] - two[1]) / two[0])
            extra = best(key)
        for i, j in enumerate(path):
            nodes[b, i] = j
            out[b, i] = extra if i + 1 == len(path) else int(tokens[b, path[i + 1]])
        count[b] = len(path) - 1
    return out, nodes, count, margin


def distill(logits, mask, index, top, lse=None, temperature=1.0, grad_loss=None):
    """(loss, tolerance, gradient, tolerance) in fp64; the gradient from the formula."""
    x, top = logits.cpu().double(), top.cpu().double()
    mask, index = mask.cpu(), index.cpu().long()
    B, L, V = x.shape
    loss, loss_tol = torch.zeros(B, L, dtype=torch.float64), torch.zeros(B, L, dtype=torch.float64)
    grad, grad_tol = torch.zeros_like(x), torch.zeros_like(x)
    z = 2.0 ** -22 + U * (4 * math.log2(max(2, V)) + V / 256 + 40)
    e = 152 * U
    for b in range(B):
        for t in range(L):
            if not mask[b, t]:
                continue
            row = x[b, t]
            there = [(int(v), float(top[b, t, k])) for k, v in enumerate(index[b, t]) if 0 <= int(v) < V]
            g = None if grad_loss is None else float(grad_loss[b, t])
            if torch.isnan(row).any() or not math.isfinite(float(row.max())) or \
                    any(math.isnan(s) or s == math.inf for _, s in there):
                loss[b, t] = math.nan
                grad[b, t] = math.nan
                continue
            log_q = torch.log_softmax(row / temperature, 0)
            q = log_q.exp()
            scores = torch.tensor([s / temperature for _, s in there], dtype=torch.float64)
            if lse is not None:
                weights = torch.exp(scores - float(lse[b, t]))
            elif len(there) and float(scores.max()) > -math.inf:
                weights = torch.softmax(scores, 0)
            else:
                weights = torch.zeros(len(there), dtype=torch.float64)
            p = torch.zeros(V, dtype=torch.float64)
            listed = torch.zeros(V, dtype=torch.bool)
            for (v, _), w in zip(there, weights.tolist()):
                p[v] += w
                listed[v] = True
            on = p > 0
            value = float((p[on] * (p[on].log() - log_q[on])).sum())
            size = (row - row.max()).abs() / temperature
            log_z = float(torch.logsumexp((row - row.max()) / temperature, 0))
            known = on & torch.isfinite(size)
            slack = float((p[known] * (e * (1 + (p[known].log() - log_q[known]).abs()) + z + e +
                                       4 * U * (p[known].log().abs() + size[known] + log_z))).sum())
            P = float(p.sum())
            R = max(0.0, 1.0 - P) if lse is not None else 0.0
            r = float(q[~listed].sum()) if (~listed).any() else 0.0
            rest = row[~listed]
            some = (~listed).any() and float(rest.max()) > -math.inf
            dx, off = q * P - p, (q * P + p) * 2 * (z + e)
            if R > 0 and some:
                # log r and s from the rest's own maximum: r may be below the smallest number
                # (both sums relative to the row's maximum, which may be 1e38)
                log_r = float(torch.logsumexp((rest - row.max()) / temperature, 0)) - log_z
                s = torch.where(listed, 0.0, torch.exp(log_q - log_r))
                value += R * (math.log(R) - log_r)
                slack += e * (1 + abs(math.log(R) - log_r)) + R * (z + e + 4 * U * (
                    abs(math.log(R)) + abs(log_r) + float((row.max() - rest.max()) / temperature) + log_z))
                dx = dx + R * (q - s)
                off = off + R * (q + s) * 2 * (z + e) + e * (q + s)
            elif lse is not None:
                off = off + e * q
            loss[b, t], loss_tol[b, t] = value, slack + 4 * U * abs(value) + 1e-30
            if g is not None:
                grad[b, t] = dx * g / temperature
                far = torch.nan_to_num(size, posinf=0.0) * 4 * U  # (t ln 2 = size)
                off = off + far * (q * (P + R) + (R * s if R > 0 and some else 0.0)) + 2.0 ** -126 * (P + 2 * R)
                grad_tol[b, t] = (off * abs(g) / temperature + EPS[logits.dtype] * grad[b, t].abs() * 1.001
                                  + TINY[logits.dtype])
    return loss, loss_tol, grad, grad_tol
