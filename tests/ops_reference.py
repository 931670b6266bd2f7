"""The operators on a caller's paged cache and logits, written plainly in 64 bits, and bounds of what their kernels may be off."""
import math

import torch

# largest relative error of one rounding to the type
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def pools(gen, lens, hk, page, d, dtype, layout="hnd", spare=2, fill=None):
    """Pools with the pages of every sequence in a random order, and the table (-1: none).  Rows behind a sequence's last position hold
    `fill`, or other numbers."""
    need = [-(-n // page) for n in lens]
    total, width = sum(need) + spare, max(1, max(need, default=1))
    order = torch.randperm(total, generator=gen)
    table = torch.full((len(lens), width + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (total, hk, page, d) if layout == "hnd" else (total, page, hk, d)
    out = []
    for _ in range(2):
        x = torch.randn(shape, generator=gen).to(dtype)
        x = x if layout == "hnd" else x.transpose(1, 2)
        if fill is not None:
            keep = torch.zeros(total, page, dtype=torch.bool)
            for b, n in enumerate(lens):
                for p in range(need[b]):
                    keep[table[b, p], :min(page, n - p * page)] = True
            x = torch.where(keep[:, None, :, None], x.float(), torch.tensor(fill)).to(dtype)
            if layout != "hnd":
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
        out.append(x)
    return out[0], out[1], table


def attend(q, k, v, table, lens, counts=None, causal=True, window=0, scale=None):
    """(out, lse, slack): all [batch, m, heads, ...] in 64 bits; slack bounds |out| errors of relative size one of the weights."""
    b_, m, h, d = q.shape
    hk, page = k.shape[1:3]
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full((b_, m, h), -math.inf, dtype=torch.float64)
    weight, score = torch.zeros(q.shape, dtype=torch.float64), torch.zeros((b_, m, h), dtype=torch.float64)
    for b in range(b_):
        n = min(int(lens[b]), table.shape[1] * page)
        n_q = m if counts is None else int(counts[b])
        for j in range(min(n_q, m)):
            last = n - n_q + j if causal else n - 1
            first = max(0, last - window + 1) if window else 0
            pos = [t for t in range(first, last + 1) if 0 <= int(table[b, t // page]) < k.shape[0]]
            if not pos:
                continue
            t = torch.tensor(pos)
            pages, rows = table[b].long()[t // page], t % page
            for head in range(h):
                kk, vv = k[pages, head // (h // hk), rows].double(), v[pages, head // (h // hk), rows].double()
                qq = q[b, j, head].double()
                s = scale * (kk @ qq)
                lse[b, j, head] = torch.logsumexp(s, 0)
                p = torch.exp(s - lse[b, j, head])
                out[b, j, head] = p @ vv
                weight[b, j, head] = p @ vv.abs()
                score[b, j, head] = abs(scale) * (kk.abs() @ qq.abs()).max()
    return out, lse, weight, score


def append(q, k, v, kp, vp, table, starts, counts, rope, interleaved):
    """(q_out, keys, values) and the bounds of the rotated ones before rounding."""
    d, page = k.shape[3], kp.shape[2]
    r = 0 if rope is None else 2 * rope.shape[1]
    first = torch.arange(0, r, 2) if interleaved else torch.arange(r // 2)
    second = first + 1 if interleaved else first + r // 2

    def turned(x, p):
        y, w = x.double().clone(), x.double().abs()
        if r:
            c, s = rope[p, :, 0].double(), rope[p, :, 1].double()
            a, b = y[..., first].clone(), y[..., second].clone()
            y[..., first], y[..., second] = a * c - b * s, a * s + b * c
            both = a.abs() + b.abs()
            w[..., first], w[..., second] = both, both
        return y, w
    q_out = None if q is None else torch.zeros(q.shape, dtype=torch.float64)
    q_w = None if q is None else torch.zeros(q.shape, dtype=torch.float64)
    kp, vp = kp.double().clone(), vp.double().clone()
    kw = torch.zeros_like(kp)
    for b in range(k.shape[0]):
        for j in range(k.shape[1]):
            p = int(starts[b]) + j
            if (counts is not None and j >= int(counts[b])) or (rope is not None and not 0 <= p < rope.shape[0]):
                continue
            if q is not None:
                q_out[b, j], q_w[b, j] = turned(q[b, j], p)
            if p < 0 or p // page >= table.shape[1] or not 0 <= int(table[b, p // page]) < kp.shape[0]:
                continue
            at = int(table[b, p // page])
            kp[at, :, p % page], kw[at, :, p % page] = turned(k[b, j], p)
            vp[at, :, p % page] = v[b, j].double()
    return q_out, kp, vp, q_w, kw


def logprobs(z, tokens, top, temperature):
    """(logprob, entropy, lse, ids, top_logprobs) of finite rows and rows of -infinity, in 64 bits."""
    raw, z = z.double(), z.double() / temperature
    lse = torch.logsumexp(z, -1)
    none = lse == -math.inf
    logp = torch.where(none[:, None], -math.inf, z - torch.where(none, 0.0, lse)[:, None])
    p = torch.where(none[:, None], 0.0, torch.exp(logp))
    entropy = torch.special.entr(p).sum(-1)
    has = (tokens >= 0) & (tokens < z.shape[1])
    logprob = torch.where(has, logp.gather(1, tokens.clamp(0, z.shape[1] - 1).long()[:, None])[:, 0], 0.0)
    ids = torch.sort(raw, dim=-1, descending=True, stable=True)[1][:, :top]
    return logprob, entropy, lse, ids, logp.gather(1, ids)


def logprobs_grad(z, tokens, ids, g, ge, gs, gt, temperature):
    """(gradient, bound of the size of its terms)."""
    logprob, entropy, lse, _, _ = logprobs(z, tokens, 0, temperature)
    z = z.double() / temperature
    none = lse == -math.inf
    logp = torch.where(none[:, None], -math.inf, z - torch.where(none, 0.0, lse)[:, None])
    p = torch.exp(logp)
    has = ((tokens >= 0) & (tokens < z.shape[1])).double()
    g = g.double() * has
    total = g - gs.double() + (gt.double().sum(-1) if gt is not None else 0.0)
    x = torch.where(p > 0, logp, 0.0) + entropy[:, None]
    d = -p * total[:, None] - ge.double()[:, None] * p * x
    size = p * ((g.abs() + gs.double().abs() + (gt.double().abs().sum(-1) if gt is not None else 0.0))[:, None] +
                ge.double().abs()[:, None] * (x.abs() + 1))
    d.scatter_add_(1, tokens.clamp(0, z.shape[1] - 1).long()[:, None], g[:, None])
    if gt is not None:
        d.scatter_add_(1, ids.long(), gt.double())
    d = torch.where(none[:, None], 0.0, d)
    return d / temperature, size / temperature
