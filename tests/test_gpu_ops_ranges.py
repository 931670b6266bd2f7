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
    """linear_grad of rows of one size after the other: every row's bound goes by its own size.  The weights' gradient: the rows of each size, and what fp16 steps of 2^-24 leave of a
    scaled operand next to the largest row's 2^13: for each row 2^-25 times 2^-12 of the largest |hidden| (2|g| + |g_lse|)."""
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
