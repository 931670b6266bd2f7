"""Gradients of the products where rows differ in size: what one row holds is nothing to another, padding has no part, and what the middle part holds does not leave fp16's range."""
import math

import pytest
import torch

import block_reference as ref
from block_reference import BF16, F16, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    yield ops
    ops.check()


def loss_inputs(rows, vocab, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((rows, d), generator=g, device="cuda").to(dtype)
    w = (2.0 * d ** -0.5 * torch.randn((vocab, d), generator=g, device="cuda")).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    gl, gs = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    return h, w, t, gl, gs


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab", [(6, 300), (300, 500), (70001, 200)])
@pytest.mark.parametrize("size", [2.0 ** 27, 1e30, math.inf, math.nan])
def test_gradients_of_rows_without_a_token_do_not_count(ops, dtype, rows, vocab, size):
    """Padding's gradient by its log probability, of any size, changes nothing: a bit more or less than with zeros there is as far off as any rounding."""
    h, w, t, gl, gs = loss_inputs(rows, vocab, 64, dtype, seed=1)
    t[1::3] = -1
    t[2] = vocab
    none = (t < 0) | (t >= vocab)
    g = torch.where(none, size, gl)
    r = ops.linear_logprobs(h, w, t)
    got = ops.linear_logprobs_grad(h, w, t, r, g, gs)
    want = ops.linear_logprobs_grad(h, w, t, r, torch.where(none, 0.0, gl), gs)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    few = rows <= 128
    x, bound = ref.linear_grad(h[:300], w, t[:300], 1.0, torch.where(none, 0.0, gl)[:300], gs[:300], 2 if few else 1)[0]
    near(got[0][:300], x, bound, "d_hidden")


@pytest.mark.parametrize("rows", [6, 300])
def test_rows_in_which_nothing_has_a_part_do_not_count(ops, rows):
    """A row of which every logit is -infinity has no gradient, whatever comes back for it."""
    h, w, t, gl, gs = loss_inputs(rows, 300, 64, F16, seed=2)
    w[:, 0] = -w[:, 0].abs() - 0.25
    h[1, 0] = math.inf
    r = ops.linear_logprobs(h, w, t)
    assert r.lse[1] == -math.inf
    d = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(True, False))[0]
    gl[1], gs[1] = 1e30, 1e30
    assert torch.equal(ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(True, False))[0], d)


def loss_by_size(h, w, t, temperature, gl, gs, sizes, parts):
    """linear_grad of rows of one size after the other: every row's bound goes by its own size.  The weights' gradient: the rows of each size, and for every row what fp16's steps leave of it next
    to the largest: of its gradients 2^-25, these 2^13 of the largest's, and of its hidden states, 2^-12 of which a row of 2^-12 of the largest keeps as 2^-25 at worst: with |hidden| above
    two both are less than 2^-37 of the largest |hidden| (2|g| + |g_lse|)."""
    dh, bh = torch.zeros(h.shape, dtype=torch.float64, device="cuda"), torch.zeros(h.shape, dtype=torch.float64, device="cuda")
    dw, bw = 0.0, 0.0
    kinds = sizes.unique()
    for s in kinds:
        at = sizes == s
        (x, b), (y, c) = ref.linear_grad(h[at], w, t[at], temperature, gl[at], gs[at], parts)
        dh[at], bh[at] = x, b
        dw, bw = dw + y, bw + c
    most = float((h.abs().amax(-1).double() * (2 * gl.double().abs() + gs.double().abs()) / temperature).max())
    # (the tensor core's accumulator holds all rows' sum while it takes the last of them)
    return (dh, bh), (dw, bw * len(kinds) + h.shape[0] * 2.0 ** -37 * most)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab", [(40, 700), (300, 40), (700, 900)])
@pytest.mark.parametrize("apart", [20, 30])
def test_losses_of_rows_of_unequal_size(ops, dtype, rows, vocab, apart):
    """Rows whose gradients are 2^apart apart, each as near as if it were alone."""
    h, w, t, gl, gs = loss_inputs(rows, vocab, 64, dtype, seed=3)
    sizes = 2.0 ** (apart // 2 - (torch.arange(rows, device="cuda") % 5) * (apart / 4)).floor().float()
    sizes = torch.where(torch.arange(rows, device="cuda") % 5 == 4, 2.0 ** (apart // 2 - apart), sizes)
    gl, gs = gl * sizes, gs * sizes
    few = rows <= 128 or vocab <= 64
    r = ops.linear_logprobs(h, w, t)
    got = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    for x, (want, bound), what in zip(got, loss_by_size(h, w, t, 1.0, gl, gs, sizes, 2 if few else 1), ("d_hidden", "d_weight")):
        sure = want.abs() + bound < 65000
        near(torch.where(sure, x.double(), 0.0), torch.where(sure, want, 0.0), bound, what)


@pytest.mark.parametrize("size", [1.0, 2.0 ** -12])
def test_weights_gradient_of_many_rows_in_fp16(ops, size):
    """More than 65536 rows, and a vocabulary in pieces: the sum over all of them, by chunks of rows in 64 bits."""
    rows, vocab = 70001, 2500
    h, w, t, gl, gs = loss_inputs(rows, vocab, 64, F16, seed=4)
    gl, gs = gl * size, gs * size
    r = ops.linear_logprobs(h, w, t)
    d_hidden, d_weight = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    alone = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(False, True))[1]
    want, bound, chunk = 0.0, 0.0, 20000
    for a in range(0, rows, chunk):
        (x, b), (y, c) = ref.linear_grad(h[a:a + chunk], w, t[a:a + chunk], 1.0, gl[a:a + chunk], gs[a:a + chunk])
        near(d_hidden[a:a + chunk], x, b + x.abs() * 2.0 ** -22, "d_hidden")
        want, bound = want + y, bound + c
    for x in (d_weight, alone):
        near(x, want, bound * (rows / chunk + 1), "d_weight")


# ------------------------------------------------------------------------------------------------- the gated feed-forward part

def gated_inputs(rows, ff, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, d), generator=g, device="cuda").to(dtype)
    wg, wu = ((1.5 * d ** -0.5 * torch.randn((ff, d), generator=g, device="cuda")).to(dtype) for _ in range(2))
    return x, wg, wu, torch.randn((rows, ff), generator=g, device="cuda").to(dtype)


def gated_by_size(x, wg, wu, gy, kind, sizes, parts):
    """gated_grad of rows of one size after the other, each with its own bound.  What fp16's steps leave of a row next to the largest, as for the losses, by the bound of its gradients:
    |g| |x| max(1.13 |w_up|, |w_gate|); of the row itself 2^-26 of that."""
    kinds = sizes.unique()
    norm = x.double().norm(dim=-1)
    factor = max(1.13 * float(wu.double().norm(dim=-1).max()), float(wg.double().norm(dim=-1).max()))
    bounds = gy.double().abs().amax(-1) * norm * factor
    dx, bx = torch.zeros(x.shape, dtype=torch.float64, device="cuda"), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    out = [[dx, bx], [0.0, 0.0], [0.0, 0.0]]
    for s in kinds:
        at = sizes == s
        (v, b), *more = ref.gated_grad(x[at], wg, wu, gy[at], kind, parts)
        dx[at] = v
        bx[at] = b + 2.0 ** -26 * bounds[at][:, None] * (wg.double().abs().sum(0) + wu.double().abs().sum(0))
        for o, (v, b) in zip(out[1:], more):
            o[0], o[1] = o[0] + v, o[1] + b * len(kinds)
    for o in out[1:]:
        o[1] = o[1] + x.shape[0] * 2.0 ** -37 * (1 + float(x.abs().max())) * float(bounds.max())
    return out


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("rows,ff,d", [(40, 700, 64), (300, 30, 64), (700, 515, 128)])
@pytest.mark.parametrize("top", [0, 10])
def test_gated_gradients_of_rows_of_unequal_size(ops, dtype, kind, rows, ff, d, top):
    """Rows 2^24 apart, each as near as if it were alone; rows of zeros between them."""
    x, wg, wu, gy = gated_inputs(rows, ff, d, dtype, seed=5)
    sizes = 2.0 ** (top - 6.0 * (torch.arange(rows, device="cuda") % 5))
    gy = (gy.float().clamp(-4, 4) * sizes[:, None]).to(dtype)
    gy[3::7] = 0
    got = ops.gated_feed_forward_grad(x, wg, wu, gy, kind)
    few = rows <= 128 or ff <= 32
    for v, (want, bound), what in zip(got, gated_by_size(x, wg, wu, gy, kind, sizes, 2 if few else 1), ("d_x", "d_w_gate", "d_w_up")):
        sure = want.abs() + bound < 65000
        near(torch.where(sure, v.double(), 0.0), torch.where(sure, want, 0.0), bound, what)
    assert (got[0][3::7] == 0).all()


@pytest.mark.parametrize("rows", [1, 6, 300])
@pytest.mark.parametrize("ff", [24, 200])
@pytest.mark.parametrize("size", [300.0, 30000.0])
def test_gated_gradients_of_large_up_in_fp16(ops, rows, ff, size):
    """up beyond the type's range beside a gate of ordinary size: the gradients of small g_out are finite, and are returned."""
    x, wg, wu, gy = gated_inputs(rows, ff, 64, F16, seed=6)
    x[:, 0] = size
    wg[:, 0], wu[:, 0] = 0.0, 400.0
    assert float((x.double() @ wu.double().T).abs().min()) > 2.0 ** 16
    gy = (gy.float() * 1e-4).half()
    wu[1:] *= 0.25
    got = ops.gated_feed_forward_grad(x, wg, wu, gy)
    few = rows <= 128 or ff <= 32
    some = 0
    for v, (want, bound), what in zip(got, gated_by_size(x, wg, wu, gy, "silu", torch.ones(rows, device="cuda"), 2 if few else 1), ("d_x", "d_w_gate", "d_w_up")):
        sure = want.abs() + bound < 65000
        some += int(sure.sum())
        near(torch.where(sure, v.double(), 0.0), torch.where(sure, want, 0.0), bound, what)
    assert some > 0


def test_gated_gradients_of_ends_of_the_type(ops):
    """The largest and the smallest numbers of fp16 in every place, weights of zeros, one weight that is infinite."""
    x, wg, wu, gy = gated_inputs(140, 72, 64, F16, seed=7)
    for scale_x, scale_w, scale_g in ((2.0 ** -24, 1.0, 1.0), (1.0, 2.0 ** -24, 1.0), (1.0, 1.0, 2.0 ** -24), (2.0 ** 13, 2.0 ** -13, 2.0 ** 13), (2.0 ** -13, 2.0 ** 13, 1.0)):
        a = [(t.float() * s).half() for t, s in ((x, scale_x), (wg, scale_w), (wu, scale_w), (gy, scale_g))]
        for v, (want, bound), what in zip(ops.gated_feed_forward_grad(*a), gated_by_size(*a, "silu", torch.ones(140, device="cuda"), 1), ("d_x", "d_w_gate", "d_w_up")):
            sure = want.abs() + bound < 65000
            near(torch.where(sure, v.double(), 0.0), torch.where(sure, want, 0.0), bound, what)
    zero = torch.zeros_like(wg)
    for v in ops.gated_feed_forward_grad(x, zero, zero, gy):
        assert (v == 0).all()
    for v in ops.gated_feed_forward_grad(torch.zeros_like(x), wg, wu, gy):
        assert (v == 0).all()
    w2 = wu.clone()
    w2[5, 3] = math.inf
    d = ops.gated_feed_forward_grad(x, wg, w2, gy)
    clean = ops.gated_feed_forward_grad(x, wg, wu, gy)
    keep = torch.arange(72, device="cuda") != 5
    bound = gated_by_size(x, wg, wu, gy, "silu", torch.ones(140, device="cuda"), 1)
    assert not d[1][5].isfinite().any()
    for i in (1, 2):
        near(d[i][keep], bound[i][0][keep], bound[i][1][keep], "d_w")
        assert clean[i].isfinite().all()


# --------------------------------------------------------------------------------------------------- logits in the hundreds

def shifted(rows, vocab, dtype, common, seed, apart=0.0):
    """Logits that are `common` and some eighths, exactly: whole numbers of hidden states and weights; the given token's is `apart` above.  The third column is the token's own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h, w = torch.zeros((rows, 64), device="cuda"), torch.zeros((vocab, 64), device="cuda")
    h[:, 0], w[:, 0] = common, 1.0
    h[:, 1], w[:, 1] = 1.0, torch.randint(-16, 17, (vocab,), generator=g, device="cuda") / 8
    w[0, 1] += apart
    w[0, 2] = 1.0
    return h.to(dtype), w.to(dtype), torch.zeros(rows, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [3, 40, 300])
@pytest.mark.parametrize("vocab,apart", [(1, 0.0), (2, 0.0), (50, 12.0), (5000, 24.0), (5000, 0.0)])
@pytest.mark.parametrize("common,temperature", [(240.0, 1.0), (-112.0, 0.7), (240.0, 0.25)])
def test_what_all_logits_have_in_common_does_not_matter(ops, dtype, rows, vocab, apart, common, temperature):
    """Log probabilities are no larger than zero and off by their own size's roundings, whatever the logits' size: differences to the maximum by 2^-23 (the factor's, the product's), exponentials
    by 2^-22, their sum by one rounding for each 64 and 40 more, its logarithm by 2^-23 of itself.  lse is off by that and its own rounding.  A token's gradient is g (1 - p)."""
    h, w, t = shifted(rows, vocab, dtype, common, 8, apart)
    z = h.double() @ w.double().T / temperature
    lse = torch.logsumexp(z, -1)
    top = z.amax(-1)
    want = (z - top[:, None])[:, 0] - torch.log(torch.exp(z - top[:, None]).sum(-1))
    # (of the sum, 2^-22 for the exponentials but the maximum's, whose argument is what a rounding of 432 left)
    slack = (1 - want.exp()) * ((z.max() - z.min()) * 2.0 ** -23 + 2.0 ** -22) + (vocab / 64 + 40) * 2.0 ** -24 * (vocab > 1) + 2.0 ** -22 + want.abs() * 2.0 ** -22
    r = ops.linear_logprobs(h, w, t, temperature)
    assert (r.logprob <= 0).all()
    near(r.logprob, want, slack, "logprob")
    near(r.lse, lse, slack + (lse - top).abs() * 2.0 ** -22 + lse.abs() * 2.0 ** -24, "lse")
    g = torch.linspace(0.5, 2.0, rows, device="cuda")
    gs = torch.linspace(-0.25, 0.25, rows, device="cuda")
    with torch.no_grad():
        d = ops.linear_logprobs_grad(h, w, t, r, g, gs, temperature, need=(True, False))[0]
    p = want.exp()
    own = (-torch.expm1(want) * g + p * gs) / temperature
    # the element: logprob's error, the exponentials' 2^-23, the products'; rounded to dtype (in two parts of up to 128 rows) in the middle and in the end; fp16's steps next to 2^13
    parts = 2 if rows <= 128 or vocab <= 64 else 1
    bound = ((slack + 2.0 ** -22) * (p * (g + gs.abs())) + own.abs() * temperature * 2.0 ** -22) / temperature
    bound = bound + ref.UNIT[dtype] ** parts * own.abs() + 2.0 ** -26 * (2 * g + gs.abs()) / temperature * (dtype is F16) + ref.UNIT[dtype] * own.abs() + ref.TINY[dtype]
    near(d[:, 2], own, bound * 1.01, "d_hidden")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,d", [(3, 300, 2048), (100, 700, 4096), (300, 60, 4096), (7, 130, 8200)])
def test_probabilities_of_long_sums_of_few_rows_add_up_to_one(ops, dtype, rows, vocab, d):
    """Products of one sign, whose sums are cut off the same way step after step: the gradient by the logits adds up to g_lse, as near as sums of 512 steps at a time are (the first column of the
    weights, which no hidden state meets, adds it up)."""
    g = torch.Generator(device="cuda").manual_seed(9)
    h, w = (torch.rand(s, generator=g, device="cuda") + 0.5 for s in ((rows, d), (vocab, d)))
    h, w = h.to(dtype), (w * 20 / d).to(dtype)
    h[:, 0], w[:, 0] = 0.0, 1.0
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    gl, gs = torch.rand(rows, generator=g, device="cuda") + 0.5, torch.zeros(rows, device="cuda")
    r = ops.linear_logprobs(h, w, t)
    logprob, lse, z, b_logprob, b_lse, off = ref.linear(h, w, t, 1.0, few=True)
    near(r.lse, lse, b_lse, "lse")
    with torch.no_grad():
        d_hidden = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(True, False))[0]
    # dz by what z and lse are off, two parts of the type, fp16's steps next to 2^13; their sum on the tensor core, both parts
    p = (z - lse[:, None]).exp()
    size = (p.sum(-1) + 1) * gl
    slack = (p * (off + b_lse[:, None] + 2.0 ** -20).expm1()).sum(-1) * gl + ref.UNIT[dtype] ** 2 * size + vocab * 2.0 ** -26 * 2 * gl * (dtype is F16)
    slack = slack + size * (-(-vocab // 16) + 2) * 2.0 ** -23 * 2
    near(d_hidden[:, 0], torch.zeros(rows, device="cuda"), slack, "sum of the gradient by the logits")


@pytest.mark.parametrize("rows", [5, 40, 300])
def test_log_probabilities_may_be_masked_in_place(ops, rows):
    """The backward pass needs none of what the caller writes to."""
    h, w, t, gl, _ = loss_inputs(rows, 300, 64, BF16, seed=10)
    h.requires_grad_()
    w.requires_grad_()
    mask = (torch.arange(rows, device="cuda") % 3 > 0).float()
    r = ops.linear_logprobs(h, w, t)
    want = torch.autograd.grad((r.logprob * mask * gl).sum(), [h, w])
    r = ops.linear_logprobs(h, w, t)
    r.logprob.mul_(mask * gl)
    got = torch.autograd.grad(r.logprob.sum(), [h, w])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows,ff", [(7, 90), (300, 24), (300, 515), (9001, 40)])
@pytest.mark.parametrize("need", [(True, False), (False, True)])
def test_some_gradients_of_rows_of_unequal_size_in_fp16(ops, rows, ff, need):
    """Each gradient by itself, where the others' operands are not made."""
    x, wg, wu, gy = gated_inputs(rows, ff, 64, F16, seed=11)
    sizes = 2.0 ** (-5.0 * (torch.arange(rows, device="cuda") % 5))
    gy = (gy.float().clamp(-4, 4) * sizes[:, None]).half()
    got = ops.gated_feed_forward_grad(x, wg, wu, gy, need=(need[0], need[1], need[1]))
    for v, (want, bound), n in zip(got, gated_by_size(x, wg, wu, gy, "silu", sizes, 2 if rows <= 128 or ff <= 32 else 1), (need[0], need[1], need[1])):
        assert n or v is None
        if n:
            near(v, want, bound, "gradient of the gated part")
    h, w, t, gl, gs = loss_inputs(rows, ff, 64, F16, seed=12)
    gl, gs = gl * sizes, gs * sizes
    r = ops.linear_logprobs(h, w, t)
    got = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=need)
    for v, (want, bound), n in zip(got, loss_by_size(h, w, t, 1.0, gl, gs, sizes, 2 if rows <= 128 or ff <= 64 else 1), need):
        assert n or v is None
        if n:
            near(v, want, bound, "gradient of the log probabilities")
