"""Log probabilities from hidden states, the gated feed-forward part and head norms with rotation, written plainly in 64 bits, each with a bound of what a kernel may be
off.  The bounds count roundings: a rounding to a type is off by half a step (UNIT), the tensor core cuts an accumulator off after every sixteen products
(2^-23 of what it holds, which the products' absolute sum bounds), an fp32 operation is off by 2^-24, the hardware's exponential, reciprocal and root by 2^-22."""
import math

import torch

from ops_reference import TINY, UNIT

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def product(a, b, few=False):
    """a b^T in 64 bits, and what a sum of its products on the tensor core may be off; few: 512 products there at most, these sums in fp32."""
    s, steps = a.abs() @ b.abs().T, -(-a.shape[1] // 16)
    return a @ b.T, s * (min(steps, 32) + steps / 64 + 3 if few else steps + 2) * 2.0 ** -23


def near(got, want, bound, what):
    """Equal where one is not finite, within the bound elsewhere."""
    got, want = got.detach().double(), want.double()
    bound = bound.expand_as(want)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want) & torch.isfinite(bound)
    odd = ~torch.isfinite(want)
    assert torch.equal(got.isnan()[odd], want.isnan()[odd]) and torch.equal(got[odd & ~want.isnan()], want[odd & ~want.isnan()]), what
    off = (got - want).abs()[fine]
    over = ~(off <= bound[fine])
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} beyond the bound, worst {float((off / bound[fine]).max()):.3g} of it"


def stored(x, slack, dtype):
    """Bound of a number that is off by `slack` and rounded to dtype."""
    return slack + UNIT[dtype] * (x.abs() + slack) + TINY[dtype]


# ------------------------------------------------------------------------------------------ log probabilities from hidden states

def linear(hidden, weight, tokens, temperature, few=False):
    """(logprob, lse, z, bound of the first, of the second, of z); few: rows or tokens that one CTA's tiles are as many as."""
    z, slack = product(hidden.double(), weight.double(), few)
    z, slack = z / temperature, slack / temperature
    size = torch.where(torch.isfinite(z), z.abs(), 0.0)
    # z log2(e) / T and its difference to the maximum, the exponential, a sum of v of them (by threads, parts and joins: at most v / 64 + 40 one after the other)
    slack = slack + size * 2.0 ** -22
    off = slack.amax(-1) + size.amax(-1) * 2.0 ** -22 + (z.shape[1] / 64 + 40) * 2.0 ** -24 + 2.0 ** -21
    lse = torch.logsumexp(z, -1)
    have = (tokens >= 0) & (tokens < weight.shape[0])
    at = tokens.clamp(0, weight.shape[0] - 1).long()[:, None]
    logprob = torch.where(have, z.gather(1, at)[:, 0] - lse, 0.0)
    off_lse = off + lse.abs() * 2.0 ** -23
    return logprob, lse, z, torch.where(have, slack.gather(1, at)[:, 0] + off_lse + logprob.abs() * 2.0 ** -24, 0.0), off_lse, slack


def linear_grad(hidden, weight, tokens, temperature, g, g_lse, parts=1):
    """((d_hidden, bound), (d_weight, bound)); parts: of dtype that the gradients by the logits are held in"""
    dtype = hidden.dtype
    logprob, lse, z, _, off_lse, off_z = linear(hidden, weight, tokens, temperature)
    rows = z.shape[0]
    none = torch.zeros(rows, dtype=torch.float64, device=z.device)
    have = (tokens >= 0) & (tokens < weight.shape[0]) & (lse > -math.inf)
    g = torch.where(have, none if g is None else g.double(), 0.0)
    s = torch.where(lse > -math.inf, none if g_lse is None else g_lse.double(), 0.0)
    p = torch.exp(z - torch.where(lse > -math.inf, lse, 0.0)[:, None])
    dz = -p * (g - s)[:, None]
    # p: the exponent is off by what z and lse are off, by their sizes' roundings; three more operations
    rel = off_z + off_lse[:, None] + (z.abs().nan_to_num(0, 0, 0) + lse.abs().nan_to_num(0, 0, 0)[:, None]) * 2.0 ** -22 + 2.0 ** -20
    # (the hardware's exponential is zero below 2^-126)
    slack = dz.abs() * rel.expm1() + 2.0 ** -126 * (g - s).abs()[:, None]
    dz[have.nonzero()[:, 0], tokens[have].long()] += g[have]
    dz, slack = dz / temperature, slack / temperature + dz.abs() / temperature * 2.0 ** -22
    # rounded to dtype, and with two parts what that left again; fp16 scaled so that the largest possible element is 2^13 at least
    most = float(((2 * g.abs() + s.abs()) / temperature).nan_to_num(0, 0, 0).amax()) if rows else 0.0
    floor = TINY[dtype] * (max(most, 2.0 ** -100) * 2.0 ** -13 if dtype is F16 else 1.0)
    slack = slack + UNIT[dtype] ** parts * (dz.abs() + slack) + floor
    out = []
    for a, b, bound in ((dz, weight.double().T, slack), (dz.T, hidden.double().T, slack.T)):
        x, more = product(a, b)
        more = more * (2 if parts > 1 else 1)        # (both parts' products, one after the other)
        out.append((x, stored(x, more + bound @ b.abs().T, dtype)))
    return out


# ---------------------------------------------------------------------------------------------------- the gated feed-forward part

def activation(g, kind):
    """act, act' and act'' bounds"""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


# the activations and their derivatives are no steeper than these (silu' <= 1.1, silu'' <= 0.5; gelu' <= 1.13, gelu'' <= 0.8)
STEEP, STEEPER = 1.13, 0.8


def gated(x, w_gate, w_up, kind):
    """(out, bound, and what its gradient needs)"""
    gate, off_g = product(x.double(), w_gate.double())
    up, off_u = product(x.double(), w_up.double())
    a, da = activation(gate, kind)
    # six operations of the hardware; Phi is off by 1.5e-7, half of erfc's; an exponent of g log2(e), or g^2 log2(e) / 2, is off by its own rounding
    off_a = STEEP * off_g + gate.abs() * (a.abs() / gate.abs().clamp(min=1e-30) + 1) * 2.0 ** -21 + (gate.abs() * 1.5e-7 if kind == "gelu" else 0.0)
    out = a * up
    return out, stored(out, off_a * up.abs() + (a.abs() + off_a) * off_u + out.abs() * 2.0 ** -22, x.dtype), (gate, up, a, da, off_g, off_u, off_a)


def gated_grad(x, w_gate, w_up, grad, kind, parts=1):
    dtype = x.dtype
    _, _, (gate, up, a, da, off_g, off_u, off_a) = gated(x, w_gate, w_up, kind)
    gy = grad.double()
    off_da = STEEPER * off_g + (1 + gate.abs()) * 2.0 ** -20 + (1.5e-7 if kind == "gelu" else 0.0)
    d_gate, d_up = gy * up * da, gy * a
    slack_g = gy.abs() * (up.abs() * off_da + (da.abs() + off_da) * off_u) + d_gate.abs() * 2.0 ** -22
    slack_u = gy.abs() * off_a + d_up.abs() * 2.0 ** -23
    fine = gy[torch.isfinite(gy)].abs()
    most = float(fine.max()) if fine.numel() else 0.0
    floor = TINY[dtype] * (max(most, 2.0 ** -100) if dtype is F16 else 1.0)        # (scaled so that the largest is 1 or more)
    slack_g, slack_u = (s + UNIT[dtype] ** parts * (d.abs() + s) + floor for s, d in ((slack_g, d_gate), (slack_u, d_up)))
    wg, wu, xx = w_gate.double(), w_up.double(), x.double()
    both, off = product(torch.cat([d_gate, d_up], 1), torch.cat([wg, wu], 0).T)
    out = [(both, stored(both, off * parts + slack_g @ wg.abs() + slack_u @ wu.abs(), dtype))]
    for d, s in ((d_gate, slack_g), (d_up, slack_u)):
        v, off = product(d.T, xx.T)
        out.append((v, stored(v, off * parts + s.T @ xx.abs(), dtype)))
    return out


# ------------------------------------------------------------------------------------------------- head norms with the rotation

def turned(x, cs, interleaved, back=False):
    """x [..., d] turned by cs [..., half, 2], and the sizes that the turning's roundings go by."""
    half = cs.shape[-2]
    c, s = cs[..., 0], cs[..., 1] * (-1 if back else 1)
    i = torch.arange(half, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y, size = x.clone(), x.abs()
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
    return y, size


def angles(rope, positions, like):
    """(cs [batch, m, 1, half, 2], live [batch, m, 1, 1])"""
    batch, m = like.shape[:2]
    pos = torch.arange(m, device=like.device).expand(batch, m) if positions is None else positions.long()
    if rope is None:
        return torch.zeros((batch, m, 1, 0, 2), dtype=torch.float64, device=like.device), torch.ones((batch, m, 1, 1), dtype=torch.bool, device=like.device)
    live = (pos >= 0) & (pos < rope.shape[0])
    return rope.double()[pos.clamp(0, rope.shape[0] - 1)][:, :, None], live[..., None, None]


# roundings of a head's root mean square: up to 32 squares one after the other, five sums across lanes, the root
NORM = 45 * 2.0 ** -24 + 2.0 ** -22


def norm(x, gain, rope, positions, eps, interleaved, dtype=None):
    cs, live = angles(rope, positions, x)
    xd = x.double()
    r = torch.rsqrt(xd.pow(2).mean(-1, keepdim=True) + eps)
    y, size = turned(xd * r * gain.double(), cs, interleaved)
    y, size = torch.where(live, y, 0.0), torch.where(live, size, 0.0)
    return y, stored(y, size * (NORM + 6 * 2.0 ** -24), dtype or x.dtype)


def norm_grad(x, gain, grad, rope, positions, eps, interleaved):
    """((dx, bound), (d_gain, bound))"""
    cs, live = angles(rope, positions, x)
    xd, g = x.double(), gain.double()
    r = torch.rsqrt(xd.pow(2).mean(-1, keepdim=True) + eps)
    u, size = turned(grad.double(), cs, interleaved, back=True)
    w, wide = u * g, size * g.abs()
    f = r * r * (w * xd).mean(-1, keepdim=True)
    off = r * r * (wide * xd.abs()).mean(-1, keepdim=True)
    dx = torch.where(live, r * (w - xd * f), 0.0)
    slack = torch.where(live, r * (wide + xd.abs() * off) * (4 * NORM + 16 * 2.0 ** -24), 0.0)
    terms = torch.where(live, (u * xd * r), 0.0).flatten(0, 2)
    sizes = torch.where(live, (size * xd.abs() * r), 0.0).flatten(0, 2)
    d_gain = terms.sum(0)
    # sums one after the other: at most all of the rows
    return (dx, stored(dx, slack, x.dtype)), (d_gain, stored(d_gain, sizes.sum(0) * (2 * NORM + min(terms.shape[0], 4000) * 2.0 ** -24), gain.dtype))
