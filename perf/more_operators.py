"""Cases of the operators that a decoder's block is trained and served with: log probabilities of given tokens straight from hidden states
(`likelihood`, with their gradient `loss`), the gated feed-forward part (`gated`, with its gradient `gated train`), norms of queries and
keys for each head together with the rotation of the positions, for training (`norm train`) and into a paged cache (`norm append`).

`run` computes them with elementary torch operations in 32 bits, or, where `own` is set, through `paper_2507_23777_b200.ops`.
"""
import math

import torch

own = False

THETA = 10000.0
EPS = 1e-6
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


# --------------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # the rows of one verified window of four drafts; the smallest product, latency counts
        dict(name="likelihood window", op="likelihood", rows=5, vocab=4096, d=1024, temp=1.0, dtype="bf16"),
        # a serving batch over a large vocabulary of odd size
        dict(name="likelihood batch", op="likelihood", rows=96, vocab=131071, d=1024, temp=0.7, dtype="fp16"),
        # an iteration of fitting a decoding head over the mesh vocabulary
        dict(name="loss mesh vocabulary", op="loss", rows=4096, vocab=4096, d=1024, temp=1.0, dtype="bf16"),
        # training over a text-sized vocabulary: the logits alone would be 1 GB
        dict(name="loss large vocabulary", op="loss", rows=8192, vocab=32003, d=2048, temp=1.0, dtype="bf16"),
        # ragged sizes, a scaled loss
        dict(name="loss ragged", op="loss", rows=1999, vocab=5003, d=768, temp=1.3, dtype="fp16"),
        # a window of four drafts through a layer
        dict(name="gated window", op="gated", rows=5, d=1024, ff=4096, act="silu", dtype="bf16"),
        # a prompt through a wide layer
        dict(name="gated prompt", op="gated", rows=4001, d=2048, ff=8192, act="silu", dtype="fp16"),
        # a training batch of four sequences of 2048
        dict(name="gated train", op="gated train", rows=8192, d=1024, ff=4096, act="silu", dtype="bf16"),
        # ragged sizes, the other activation
        dict(name="gated train ragged", op="gated train", rows=2047, d=768, ff=2051, act="gelu", dtype="fp16"),
        # what every layer of a decoding step appends for one mesh
        dict(name="norm append window", op="norm append", batch=1, m=5, heads=16, kv_heads=16, d=64, page=64, start=1000, rot=64, inter=False,
             ragged=False, src="bf16", dtype="fp16"),
        # a training batch, grouped heads
        dict(name="norm train grouped", op="norm train", batch=4, m=2048, heads=32, kv_heads=8, d=128, rot=128, inter=False, ragged=False,
             src="bf16"),
        # sequences of unequal place, 32 bits, half of every head rotated in neighbouring pairs
        dict(name="norm train fp32", op="norm train", batch=3, m=1001, heads=16, kv_heads=16, d=64, rot=32, inter=True, ragged=True,
             src="fp32"),
    ]


def _spread(rng, low, high):
    """A whole number from low to high, even over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["likelihood", "loss", "loss", "gated", "gated train", "gated train", "norm append", "norm train"])
    dtype = rng.choice(["bf16", "fp16"])
    if op in ("likelihood", "loss"):
        d = 8 * _spread(rng, 8, 256)
        vocab = _spread(rng, 50, 150_000 if op == "likelihood" else 50_000)
        rows = _spread(rng, 1, max(1, min(512 if op == "likelihood" else 8192, 250_000_000_000 // (vocab * d))))
        return dict(op=op, rows=rows, vocab=vocab, d=d, temp=rng.choice([1.0, 1.0, 0.6, 1.3]), dtype=dtype)
    if op in ("gated", "gated train"):
        d, ff = 8 * _spread(rng, 8, 256), _spread(rng, 64, 8192)
        rows = _spread(rng, 1, max(1, min(8192, 60_000_000_000 // (ff * d))))
        return dict(op=op, rows=rows, d=d, ff=ff, act=rng.choice(["silu", "silu", "gelu"]), dtype=dtype)
    d = rng.choice([32, 64, 64, 96, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 7])
    batch = _spread(rng, 1, 64)
    src = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    m = _spread(rng, 1, max(1, min(4096, 40_000_000 // ((heads + kv_heads) * d * batch))))
    case = dict(op=op, batch=batch, m=m, heads=heads, kv_heads=kv_heads, d=d, rot=rng.choice([d, d, d // 2]), inter=rng.random() < 0.3,
                ragged=rng.random() < 0.5, src=src)
    if op == "norm append":
        case.update(page=rng.choice([16, 32, 64, 128]), start=_spread(rng, 1, 2000) - 1, dtype=src if src != "fp32" else rng.choice(["fp32", "fp16"]))
    return case


def _counts(case):
    """New tokens of every sequence of an append."""
    b, m = case["batch"], case["m"]
    return [m] * b if not case["ragged"] or m == 1 else [max(1, m * (i + 1) // b) for i in range(b)]


def work(case):
    op = case["op"]
    if op in ("likelihood", "loss"):
        n, v, d = case["rows"], case["vocab"], case["d"]
        e = SIZE[case["dtype"]]
        once = (n + v) * d * e + 16 * n
        return {"bytes": once, "flops": 2 * n * v * d} if op == "likelihood" else {"bytes": 2 * once, "flops": 6 * n * v * d}
    if op in ("gated", "gated train"):
        n, f, d = case["rows"], case["ff"], case["d"]
        e = SIZE[case["dtype"]]
        read, out = (n + 2 * f) * d * e, n * f * e
        return {"bytes": read + out, "flops": 4 * n * f * d} if op == "gated" else {"bytes": 2 * (read + out), "flops": 12 * n * f * d}
    h, k, d, e = case["heads"], case["kv_heads"], case["d"], SIZE[case["src"]]
    if op == "norm append":
        t = sum(_counts(case))
        return {"bytes": t * d * (2 * h * e + 2 * k * (e + SIZE[case["dtype"]])), "flops": t * (h + k) * (5 * d + 3 * case["rot"])}
    t = case["batch"] * case["m"]
    return {"bytes": t * (h + k) * d * e * 4, "flops": t * (h + k) * (16 * d + 6 * case["rot"])}


# ------------------------------------------------------------------------------------------------------------- their inputs

def _angles(n, rot):
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * \
        THETA ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _heads(case, gen):
    """Queries, keys and values as a joint projection leaves them, side by side; heads of unequal size, as projections have them."""
    b, m, h, hk, d = (case[n] for n in ("batch", "m", "heads", "kv_heads", "d"))
    qkv = torch.randn((b, m, (h + 2 * hk) * d), generator=gen, device="cuda")
    qkv *= torch.exp(torch.randn((1, 1, h + 2 * hk, 1), generator=gen, device="cuda").expand(-1, -1, -1, d).reshape(1, 1, -1))
    qkv = qkv.to(TYPES[case["src"]])
    q, k, v = (x.view(b, m, -1, d) for x in qkv.split([h * d, hk * d, hk * d], -1))
    gains = [1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
    return dict(q=q, new_k=k, new_v=v, q_gain=gains[0], k_gain=gains[1])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, st = case["op"], dict(case=case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if op in ("likelihood", "loss"):
        n, v, d, kind = case["rows"], case["vocab"], case["d"], TYPES[case["dtype"]]
        st["weight"] = (2.0 * d ** -0.5 * normal(v, d)).to(kind)
        st["tokens"] = torch.randint(0, v, (n,), generator=gen, device="cuda")
        # normalised hidden states; the given token is mostly a likely one
        lean = torch.rand((n, 1), generator=gen, device="cuda")
        h = normal(n, d) + 1.5 * lean * st["weight"][st["tokens"]].float()
        st["hidden"] = (h * torch.rsqrt((h * h).mean(-1, keepdim=True))).to(kind)
        if op == "loss":
            st["tokens"][::17] = -1          # padding: places without a token
            scale = 1024.0 if case["dtype"] == "fp16" else 1.0          # fp16 training scales its loss
            st["g"] = scale / n * -torch.rand(n, generator=gen, device="cuda")
            st["g_lse"] = scale / n * 0.1 * normal(n)
        return st
    if op in ("gated", "gated train"):
        n, f, d, kind = case["rows"], case["ff"], case["d"], TYPES[case["dtype"]]
        st["x"] = normal(n, d).to(kind)
        st["w_gate"], st["w_up"] = ((1.5 * d ** -0.5 * normal(f, d)).to(kind) for _ in range(2))
        if op == "gated train":
            st["g"] = (normal(n, f) * (0.05 if case["dtype"] == "fp16" else 1.0 / n)).to(kind)
        return st
    st.update(_heads(case, gen))
    b, m, h, hk, d = (case[n] for n in ("batch", "m", "heads", "kv_heads", "d"))
    if op == "norm append":
        p = case["page"]
        mix = torch.randperm(b, generator=gen, device="cuda").cpu()
        starts = torch.tensor([case["start"] * (i + 1) // b if case["ragged"] else case["start"] for i in range(b)])[mix]
        counts = torch.tensor(_counts(case))[mix]
        need = [-(-(int(s) + m) // p) for s in starts]
        total = sum(need) + 3
        order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
        st["table"] = torch.full((b, max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            st["table"][i, :n] = order[at:at + n]
            at += n
        st["k"], st["v"] = (normal(total, hk, p, d).to(TYPES[case["dtype"]]) for _ in range(2))
        st["starts"], st["counts"] = starts.to(torch.int32).cuda(), counts.to(torch.int32).cuda() if case["ragged"] else None
        st["rope"] = _angles(int(starts.max()) + m + 1, case["rot"])
        st["q_out"] = torch.empty((b, m, h, d), dtype=TYPES[case["src"]], device="cuda")
        if own:
            # the handle of the pool, which a program makes once
            from paper_2507_23777_b200 import ops
            st["cache"] = ops.PagedCache(st["k"], st["v"])
        return st
    # sequences that begin at places of their own (ragged), or all at 0
    first = torch.randint(0, 500, (b, 1), generator=gen, device="cuda") if case["ragged"] else torch.zeros((b, 1), dtype=torch.int64, device="cuda")
    st["positions"] = (first + torch.arange(m, device="cuda")).to(torch.int32)
    st["rope"] = _angles(m + 500, case["rot"])
    st["g_q"], st["g_k"] = (normal(b, m, n, d).to(TYPES[case["src"]]) for n in (h, hk))
    return st


# ---------------------------------------------------------------------------------------------------------- the plain forms

def _likelihood(st):
    t = st["tokens"]
    z = torch.matmul(st["hidden"].float(), st["weight"].float().T) * (1.0 / st["case"]["temp"])
    top = z.amax(-1, keepdim=True)
    lse = (torch.log(torch.exp(z - top).sum(-1, keepdim=True)) + top)[:, 0]
    logprob = torch.where(t >= 0, z.gather(1, t.clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    return logprob, lse, z


def _loss(st):
    t = st["tokens"]
    logprob, lse, z = _likelihood(st)
    g = torch.where(t >= 0, st["g"], 0.0)
    d = torch.exp(z - lse[:, None]) * (st["g_lse"] - g)[:, None]
    d.scatter_add_(1, t.clamp(min=0)[:, None], g[:, None])
    d = d * (1.0 / st["case"]["temp"])
    kind = st["hidden"].dtype
    return logprob, lse, torch.matmul(d, st["weight"].float()).to(kind), torch.matmul(d.T, st["hidden"].float()).to(kind)


def _activation(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    c = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * c, c + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _gated(st):
    x = st["x"].float()
    wg, wu = st["w_gate"].float(), st["w_up"].float()
    gate, up = torch.matmul(x, wg.T), torch.matmul(x, wu.T)
    a, da = _activation(gate, st["case"]["act"])
    kind = st["x"].dtype
    out = (a * up).to(kind)
    if st["case"]["op"] == "gated":
        return out
    g = st["g"].float()
    d_gate, d_up = g * up * da, g * a
    return out, (torch.matmul(d_gate, wg) + torch.matmul(d_up, wu)).to(kind), torch.matmul(d_gate.T, x).to(kind), torch.matmul(d_up.T, x).to(kind)


def _rotate(x, cs, case, back=False):
    """Rotates the first `rot` elements of every head; cs: [batch, m, rot / 2, 2]."""
    r = case["rot"]
    c, s = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
    s = -s if back else s
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["inter"] else (x[..., :r // 2], x[..., r // 2:r])
    u, w = a * c - b * s, a * s + b * c
    y = torch.stack([u, w], -1).flatten(-2) if case["inter"] else torch.cat([u, w], -1)
    return torch.cat([y, x[..., r:]], -1)


def _norm(x, gain, cs, case):
    return _rotate(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain, cs, case)


def _norm_append(st):
    case, p = st["case"], st["case"]["page"]
    b, m = case["batch"], case["m"]
    j = torch.arange(m, device="cuda")
    pos = st["starts"].long()[:, None] + j
    real = (j < (st["counts"][:, None] if st["counts"] is not None else m)).expand(b, m)[:, :, None, None]
    cs = st["rope"][pos]
    q = torch.where(real, _norm(st["q"].float(), st["q_gain"], cs, case), 0.0)
    page, row = st["table"].gather(1, pos // p).long(), pos % p
    for pool, x in ((st["k"], _norm(st["new_k"].float(), st["k_gain"], cs, case)), (st["v"], st["new_v"].float())):
        there = pool[page, :, row]          # [batch, m, kv heads, d]; what a place holds stays where there is no new token
        pool[page, :, row] = torch.where(real, x.to(pool.dtype), there)
    return q.to(st["q"].dtype), st["k"], st["v"]


def _norm_grad(x, gain, g, cs, case):
    u = _rotate(g, cs, case, back=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    w = u * gain
    return r * (w - x * (r * r) * (w * x).mean(-1, keepdim=True)), (u * x * r).sum((0, 1, 2))


def _norm_train(st):
    case, kind = st["case"], st["q"].dtype
    cs = st["rope"][st["positions"].long()]
    q, k = st["q"].float(), st["new_k"].float()
    dq, dq_gain = _norm_grad(q, st["q_gain"], st["g_q"].float(), cs, case)
    dk, dk_gain = _norm_grad(k, st["k_gain"], st["g_k"].float(), cs, case)
    return (_norm(q, st["q_gain"], cs, case).to(kind), _norm(k, st["k_gain"], cs, case).to(kind), dq.to(kind), dk.to(kind), dq_gain, dk_gain)


def _own(st):
    from paper_2507_23777_b200 import ops
    case = st["case"]
    op = case["op"]
    if op in ("likelihood", "loss"):
        r = ops.linear_logprobs(st["hidden"], st["weight"], st["tokens"], temperature=case["temp"])
        if op == "likelihood":
            return r.logprob, r.lse
        d_hidden, d_weight = ops.linear_logprobs_grad(st["hidden"], st["weight"], st["tokens"], r, grad_logprob=st["g"], grad_lse=st["g_lse"],
                                                      temperature=case["temp"])
        return r.logprob, r.lse, d_hidden, d_weight
    if op in ("gated", "gated train"):
        out = ops.gated_feed_forward(st["x"], st["w_gate"], st["w_up"], activation=case["act"])
        if op == "gated":
            return out
        return (out, *ops.gated_feed_forward_grad(st["x"], st["w_gate"], st["w_up"], st["g"], activation=case["act"]))
    if op == "norm append":
        q = st["cache"].append(st["new_k"], st["new_v"], st["table"], st["starts"], counts=st["counts"], q=st["q"], rope=st["rope"],
                               interleaved=case["inter"], out=st["q_out"], q_gain=st["q_gain"], k_gain=st["k_gain"], eps=EPS)
        return q, st["k"], st["v"]
    more = dict(rope=st["rope"], positions=st["positions"], eps=EPS, interleaved=case["inter"])
    q, k = ops.norm_rotate(st["q"], st["new_k"], st["q_gain"], st["k_gain"], **more)
    return (q, k, *ops.norm_rotate_grad(st["q"], st["new_k"], st["q_gain"], st["k_gain"], st["g_q"], st["g_k"], **more))


def run(st):
    if own:
        return _own(st)
    op = st["case"]["op"]
    if op == "likelihood":
        return _likelihood(st)[:2]
    if op == "loss":
        return _loss(st)
    if op in ("gated", "gated train"):
        return _gated(st)
    return _norm_append(st) if op == "norm append" else _norm_train(st)


# --------------------------------------------------------------------------------------------- the definitions in 64 bits

def _exact_rows(st):
    """Straight from the definition, gradients by differentiation; a piece of the rows at a time."""
    case, t = st["case"], st["tokens"]
    train = case["op"] == "loss"
    w = st["weight"].double().requires_grad_(train)
    piece = max(1, 100_000_000 // case["vocab"])
    parts, d_weight = [], None
    for a in range(0, case["rows"], piece):
        h = st["hidden"][a:a + piece].double().requires_grad_(train)
        z = torch.einsum("rd,vd->rv", h, w) / case["temp"]
        lse = torch.logsumexp(z, -1)
        have = torch.nonzero(t[a:a + piece] >= 0)[:, 0]
        picked = z[have, t[a:a + piece][have]] - lse[have]
        r = [torch.zeros_like(lse).index_put((have,), picked), lse]
        if train:
            total = (picked * st["g"][a:a + piece][have].double()).sum() + (lse * st["g_lse"][a:a + piece].double()).sum()
            dh, dw = torch.autograd.grad(total, [h, w])
            d_weight = dw if d_weight is None else d_weight + dw
            r.append(dh)
        parts.append([x.detach() for x in r])
    return [torch.cat(x) for x in zip(*parts)] + ([d_weight] if train else [])


def _exact_gated(st):
    train = st["case"]["op"] == "gated train"
    x, wg, wu = (st[n].double().requires_grad_(train) for n in ("x", "w_gate", "w_up"))
    gate, up = torch.einsum("rd,fd->rf", x, wg), torch.einsum("rd,fd->rf", x, wu)
    y = (torch.nn.functional.silu(gate) if st["case"]["act"] == "silu" else torch.nn.functional.gelu(gate)) * up
    return [y.detach(), *torch.autograd.grad(y, [x, wg, wu], st["g"].double())] if train else y


def _exact_turn(y, pos, case):
    r = case["rot"]
    half = torch.arange(r // 2, device="cuda")
    first, second = (2 * half, 2 * half + 1) if case["inter"] else (half, half + r // 2)
    angle = pos.double()[..., None, None] * torch.pow(torch.tensor(THETA, dtype=torch.float64, device="cuda"), -2.0 * half.double() / r)
    w = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle)
    out = y.clone()
    out[..., first], out[..., second] = w.real, w.imag
    return out


def _exact_norm(x, gain, pos, case):
    return _exact_turn(x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["d"] + EPS) * gain, pos, case)


def _exact_append(st):
    case, p = st["case"], st["case"]["page"]
    q_out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    k, v = st["k"].double(), st["v"].double()
    for b in range(case["batch"]):
        n = int(st["counts"][b]) if st["counts"] is not None else case["m"]
        pos = torch.arange(n, device="cuda") + int(st["starts"][b])
        q_out[b, :n] = _exact_norm(st["q"][b, :n].double(), st["q_gain"].double(), pos, case)
        page, row = st["table"][b].long()[pos // p], pos % p
        k[page, :, row] = _exact_norm(st["new_k"][b, :n].double(), st["k_gain"].double(), pos, case)
        v[page, :, row] = st["new_v"][b, :n].double()
    return q_out, k, v


def _exact_train(st):
    case = st["case"]
    outs, grads, gains = [], [], []
    for x, gain, g in ((st["q"], st["q_gain"], st["g_q"]), (st["new_k"], st["k_gain"], st["g_k"])):
        x, gain = x.double().requires_grad_(), gain.double().requires_grad_()
        y = _exact_norm(x, gain, st["positions"], case)
        dx, d_gain = torch.autograd.grad(y, [x, gain], g.double())
        outs.append(y.detach())
        grads.append(dx)
        gains.append(d_gain)
    return outs + grads + gains


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] in ("likelihood", "loss"):
        return _exact_rows(st)
    if case["op"] in ("gated", "gated train"):
        return _exact_gated(st)
    return _exact_append(st) if case["op"] == "norm append" else _exact_train(st)
