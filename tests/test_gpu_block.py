"""A decoder block with norms of queries and keys, trained and served with the library's operators, and the paths of the package that call them."""
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import block_reference as ref
from conftest import gpu_cfg
from paper_2507_23777_b200 import inputs

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    yield ops
    ops.check()


class Block:
    """One block (grouped heads, norms of queries and keys, gated feed-forward) and the output projection, of bf16 weights."""

    def __init__(self, d=256, heads=8, kv_heads=2, d_head=64, ff=520, vocab=333, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(out, into):
            return (into ** -0.5 * torch.randn((out, into), generator=g, device="cuda")).to(BF16)
        self.heads, self.kv_heads, self.d_head, self.vocab = heads, kv_heads, d_head, vocab
        self.p = dict(qkv=w((heads + 2 * kv_heads) * d_head, d), o=w(d, heads * d_head), gate=w(ff, d), up=w(ff, d), down=w(d, ff), out=w(vocab, d),
                      q_gain=1 + 0.1 * torch.randn(d_head, generator=g, device="cuda"), k_gain=1 + 0.1 * torch.randn(d_head, generator=g, device="cuda"))

    def project(self, p, x):
        b, m, _ = x.shape
        return (x @ p["qkv"].T).view(b, m, -1, self.d_head).split([self.heads, self.kv_heads, self.kv_heads], 2)

    def train(self, ops, p, x, rope, tokens):
        q, k, v = self.project(p, x)
        q, k = ops.norm_rotate(q, k, p["q_gain"], p["k_gain"], rope=rope)
        a = F.scaled_dot_product_attention(*(t.transpose(1, 2) for t in (q, k, v)), is_causal=True, enable_gqa=True).transpose(1, 2).flatten(2)
        x = x + a @ p["o"].T
        x = x + ops.gated_feed_forward(x, p["gate"], p["up"]) @ p["down"].T
        return ops.linear_logprobs(x.flatten(0, 1), p["out"], tokens.flatten())

    def exact(self, p, x, rope, tokens):
        """The same in 64 bits from the definitions."""
        q, k, v = self.project(p, x)
        cs = rope.double()[:x.shape[1]][None, :, None]
        q, k = (ref.turned(t * torch.rsqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6) * g, cs, False)[0] for t, g in ((q, p["q_gain"]), (k, p["k_gain"])))
        k, v = (t.repeat_interleave(self.heads // self.kv_heads, 2) for t in (k, v))
        s = torch.einsum("bmhd,bnhd->bhmn", q, k) * self.d_head ** -0.5
        s = s.masked_fill(torch.ones(s.shape[-2:], dtype=torch.bool, device="cuda").triu(1), -math.inf)
        x = x + torch.einsum("bhmn,bnhd->bmhd", torch.softmax(s, -1), v).flatten(2) @ p["o"].T
        x = x + (F.silu(x @ p["gate"].T) * (x @ p["up"].T)) @ p["down"].T
        logp = torch.log_softmax(x.flatten(0, 1) @ p["out"].T, -1)
        t = tokens.flatten()
        return torch.where(t >= 0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)


@pytest.mark.parametrize("batch,m", [(2, 75), (1, 1), (3, 130)])
def test_a_block_is_trained(ops, batch, m):
    """Forward and backward through all of them.  Between input and loss there are ten tensors that are rounded to bf16, as many again on the way back, each by
    2^-8 of an element at most: twenty of them bound the error of a gradient's norm."""
    block = Block()
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn((batch, m, 256), generator=g, device="cuda").to(BF16)
    tokens = torch.randint(0, block.vocab, (batch, m), generator=g, device="cuda")
    if m > 1:
        tokens[0, ::5] = -1
    rope = ops.rope_table(m, 64)
    names = [*block.p, "x"]
    leaves = [t.clone().requires_grad_() for t in (*block.p.values(), x)]
    r = block.train(ops, dict(zip(names, leaves)), leaves[-1], rope, tokens)
    got = torch.autograd.grad(-r.logprob.sum() / (batch * m), leaves)
    wide = [t.double().requires_grad_() for t in (*block.p.values(), x)]
    logprob = block.exact(dict(zip(names, wide)), wide[-1], rope, tokens)
    want = torch.autograd.grad(-logprob.sum() / (batch * m), wide)
    assert float((r.logprob - logprob).detach().norm()) <= 20 * 2.0 ** -8 * float(logprob.detach().norm())
    for name, a, b in zip(names, got, want):
        if m == 1 and name in ("q_gain", "k_gain"):          # one position: the softmax is constant, and the gradient noise
            continue
        if m == 1 and name == "qkv":
            a, b = a[-2 * 64:], b[-2 * 64:]
        assert float((a.double() - b).norm()) <= 20 * 2.0 ** -8 * float(b.norm()), name


def test_a_block_is_served_as_it_was_trained(ops):
    """Windows of one to seven tokens through append with norms, attention over the pages, the gated part and the log probabilities: what the whole sequence gives at
    once, within the roundings of both (twelve each)."""
    block, m, batch = Block(seed=1), 40, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((batch, m, 256), generator=g, device="cuda").to(BF16)
    tokens = torch.randint(0, block.vocab, (batch, m), generator=g, device="cuda")
    rope = ops.rope_table(64, 64)
    with torch.no_grad():
        whole = block.train(ops, block.p, x, rope, tokens).logprob.view(batch, m)
        p = block.p
        cache = ops.PagedCache(*(torch.zeros((8, 2, 16, 64), dtype=BF16, device="cuda") for _ in range(2)))
        table = torch.randperm(8, device="cuda").view(2, 4)[:, :3].to(torch.int32).contiguous()
        got, at = [], 0
        for n in (1, 7, 1, 5, 6, 7, 4, 7, 2):
            window = x[:, at:at + n]
            q, k, v = block.project(p, window)
            starts = torch.full((batch,), at, dtype=torch.int32, device="cuda")
            q = cache.append(k, v, table, starts, q=q, rope=rope, q_gain=p["q_gain"], k_gain=p["k_gain"])
            a = cache.attend(q, table, starts + n)[0].flatten(2)
            h = window + a @ p["o"].T
            h = h + ops.gated_feed_forward(h, p["gate"], p["up"]) @ p["down"].T
            got.append(ops.linear_logprobs(h.flatten(0, 1), p["out"], tokens[:, at:at + n].flatten()).logprob.view(batch, n))
            at += n
        cache.check()
    assert at == m
    got = torch.cat(got, 1)
    assert float((got - whole).norm()) <= 24 * 2.0 ** -8 * float(whole.norm())


@pytest.fixture(scope="module")
def score(ops):
    from paper_2507_23777_b200 import score
    return score


@pytest.mark.parametrize("batch,n", [(1, 2), (3, 90)])
def test_likelihood_of_a_mesh_is_its_score(score, batch, n):
    """Hidden states rounded to bf16 once: a logit is off by 2^-8 of its products' absolute sum at most, a log probability by twice the largest of a row."""
    cfg = gpu_cfg(dtype=1, sigma=0.08, seed=3, batch=batch)
    w, cond = inputs.make_weights(cfg, random_gains=True), inputs.make_cond(cfg, batch)
    tokens = np.random.default_rng(n).integers(1, cfg["vocab"], (batch, n))
    tokens[:, 0] = cfg["bos_id"]
    s = score.Scorer(cfg, w, batch, n)
    want, got = s.score(cond, tokens), s.likelihood(cond, tokens)
    s.condition(cond)
    x = torch.as_tensor(tokens, device="cuda")
    h = torch.cat([s.hidden(x[:, a:min(a + 16, n - 1)], a) for a in range(0, n - 1, 16)], 1)
    bound = 2.0 ** -8 * (h.double().abs() @ s.W("W0").double().abs().T).amax(-1) + 1e-5
    assert ((got.lse.double() - want.lse.double()).abs() <= bound).all()
    assert ((got.logprob.double() - want.logprob.double()).abs() <= 2 * bound).all()


def test_feed_forward_parts_by_the_library(score):
    """Twice the library's own bound on logits of bf16 models, 2e-2, as for the scores of a whole sequence."""
    cfg = gpu_cfg(dtype=1, sigma=0.08, seed=4, batch=2)
    w, cond = inputs.make_weights(cfg, random_gains=True), inputs.make_cond(cfg, 2)
    tokens = np.random.default_rng(5).integers(1, cfg["vocab"], (2, 50))
    a, b = score.Scorer(cfg, w, 2, 50), score.Scorer(cfg, w, 2, 50, library_products=True)
    x, y = a.score(cond, tokens), b.score(cond, tokens)
    assert float((x.logprob - y.logprob).abs().max()) < 4e-2
    assert float((b.likelihood(cond, tokens).logprob - x.logprob).abs().max()) < 8e-2
    fp32 = gpu_cfg(dtype=0, batch=1)
    with pytest.raises(ValueError, match="bf16"):
        score.Scorer(fp32, inputs.make_weights(fp32), 1, 10, library_products=True)
    with pytest.raises(ValueError, match="bf16"):
        score.Scorer(fp32, inputs.make_weights(fp32), 1, 10).likelihood(inputs.make_cond(fp32, 1), np.array([[0, 1]]))


def test_scores_of_products_that_gave_up_are_not_returned(score):
    from paper_2507_23777_b200 import binding
    cfg = gpu_cfg(dtype=1)
    s = score.Scorer(cfg, inputs.make_weights(cfg), 1, 40, library_products=True)
    cond, tokens = inputs.make_cond(cfg, 1), np.arange(40)[None]
    want = s.likelihood(cond, tokens).logprob
    try:
        binding.load().xsm_debug_product_waits(2000, 1)
        for f in (s.likelihood, s.score):
            with pytest.raises(binding.XsmError) as e:
                f(cond, tokens)
            assert e.value.status == binding.XSM_ERR_TIMEOUT
    finally:
        binding.load().xsm_debug_product_waits(0, 0)
    assert torch.equal(s.likelihood(cond, tokens).logprob, want)


def test_heads_fitted_with_the_librarys_products(ops):
    """It runs, and its first loss is torch's: hidden states and weights rounded to bf16 once each, 2^-8 of logits of at most a few units."""
    from paper_2507_23777_b200 import fit_heads
    cfg = gpu_cfg(dtype=1, sigma=0.1, seed=11, n_draft=2)
    w = inputs.make_weights(cfg)
    rng = np.random.default_rng(0)
    seqs = [np.concatenate([[0], rng.integers(0, cfg["vocab"], 60)]) for _ in range(4)]
    conds = list(inputs.make_cond(cfg, 4))
    runs = [fit_heads.fit_from_corpus(cfg, w, seqs, conds, iters=6, lr=1e-3, eval_every=3, library_products=lib) for lib in (False, True)]
    (fa, a), (fb, b) = runs
    assert len(b["curve"]) == 3 and all(np.isfinite(c["held_out_loss"]) for c in b["curve"]) and fb.shape == fa.shape
    assert abs(a["curve"][0]["held_out_loss"] - b["curve"][0]["held_out_loss"]) < 0.05
    assert b["curve"][0]["held_out_loss"] != b["curve"][-1]["held_out_loss"]
