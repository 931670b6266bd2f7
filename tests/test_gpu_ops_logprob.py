"""Log probabilities of given tokens, entropy, alternatives and their gradient, against plain torch in 64 bits."""
import math

import pytest
import torch

import ops_reference as ref
from ops_reference import TINY, UNIT

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LOWEST = {F32: -3.4028234663852886e38, BF16: -3.3895313892515355e38, F16: -65504.0}


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    return ops


def logits(rows, vocab, dtype, seed, masked=False, step=None, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    z = spread * torch.randn((rows, vocab), generator=g)
    if step:
        z = (z / step).round() * step          # many equal ones
    t = torch.randint(0, vocab, (rows,), generator=g)
    if masked:
        gone = torch.rand((rows, vocab), generator=g) < 0.3
        gone[:, 0] = False
        z[gone] = -math.inf
    return z.to(dtype), t


def same(got, want, bound, what):
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine]) and torch.isfinite(got[fine]).all(), what
    off = (got - want).abs()[fine]
    over = off > bound.expand_as(want)[fine]
    assert not over.any(), f"{what}: {int(over.sum())} beyond the bound, worst {float((off / bound.expand_as(want)[fine]).max()):.3g} of it"


def check(ops, z, t, top, temperature, gpu=None):
    gz = z.cuda() if gpu is None else gpu
    r = ops.token_logprobs(gz, t.cuda(), top=top, temperature=temperature)
    want = ref.logprobs(z, t, top, temperature)
    v = z.shape[1]
    # Differences to the maximum and their exponentials are rounded in fp32, the exponents' size times 2^-22; sums of v terms in an order
    # of their own, by threads: (v / 256 + 40) 2^-24 of the sum, which the logarithm turns into an absolute error; the entropy sums
    # p log p, at most log v + 1 times that.
    zd = z.double() / temperature
    size = torch.where(torch.isfinite(zd), zd.abs(), 0.0).amax(-1)
    sums = (v / 256 + 40) * 2.0 ** -24
    depth = torch.where(torch.isfinite(want[2]), size, 0.0) + 1
    lse_bound = sums + depth * 2.0 ** -22
    same(r.lse, want[2], lse_bound, "lse")
    same(r.logprob, want[0], lse_bound + want[0].abs().nan_to_num(posinf=0.0) * 2.0 ** -22, "logprob")
    same(r.entropy, want[1], (math.log(v) + 2) * (2 * sums + 2.0 ** -21) + depth * 2.0 ** -21, "entropy")
    if top:
        assert torch.equal(r.top_ids.cpu().long(), want[3]), "ids"
        same(r.top_logprobs, want[4], lse_bound[:, None] + want[4].abs().nan_to_num(posinf=0.0) * 2.0 ** -22, "alternatives")
    else:
        assert r.top_ids is None and r.top_logprobs is None
    return r


def check_grad(ops, z, t, r, top, temperature, seed=0, gpu=None, in_place=False):
    g = torch.Generator().manual_seed(seed)
    rows, v = z.shape
    gl, ge, gs = (torch.randn(rows, generator=g) for _ in range(3))
    gt = torch.randn((rows, top), generator=g) if top else None
    gz = z.cuda() if gpu is None else gpu
    d = ops.token_logprobs_grad(gz, t.cuda(), r, grad_logprob=gl.cuda(), grad_entropy=ge.cuda(), grad_lse=gs.cuda(),
                                grad_top=None if gt is None else gt.cuda(), temperature=temperature, out=gz if in_place else None)
    assert d.dtype == z.dtype
    want, size = ref.logprobs_grad(z, t, None if r.top_ids is None else r.top_ids.cpu(), gl, ge, gs, gt, temperature)
    # p from the exponent z - lse: its size times 2^-22, and the error of lse and entropy; the sum of a few terms, once rounded
    zd = z.double() / temperature
    depth = torch.where(torch.isfinite(zd), zd.abs(), 0.0).amax(-1) + 2 + math.log(v)
    rel = (4 * depth * 2.0 ** -22 + 2 * (v / 256 + 40) * 2.0 ** -24 + 2.0 ** -20)[:, None]
    direct = torch.zeros_like(want).scatter_add_(1, t.clamp(0, v - 1)[:, None], gl.abs().double()[:, None])
    if top:
        direct.scatter_add_(1, r.top_ids.cpu().long(), gt.abs().double())
    same(d, want, UNIT[z.dtype] * want.abs() + rel * size + 2.0 ** -21 * direct / temperature + TINY[z.dtype], "gradient")


SIZES = [(1, 1, 1), (3, 2, 2), (4, 31, 5), (5, 50, 32), (70, 257, 1), (2, 1000, 8), (9, 1025, 20), (5, 4096, 5), (2, 4099, 32), (300, 513, 0), (3, 8192, 3),
         (4, 8193, 20), (2, 20001, 32), (17, 33000, 0), (2, 50257, 20), (1, 131071, 32), (3, 151936, 20), (1, 400001, 7)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,vocab,top", SIZES)
def test_sizes(ops, dtype, rows, vocab, top):
    for temperature in (1.0, 0.6):
        z, t = logits(rows, vocab, dtype, rows + vocab)
        if rows > 2:
            t[1], t[2] = -1, vocab
        r = check(ops, z, t, top, temperature)
        check_grad(ops, z, t, r, top, temperature)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,vocab,top", [(3, 50, 9), (400, 50, 9), (3, 5003, 20), (200, 5003, 20), (3, 40000, 32)])
def test_masked_vocabulary_and_equal_logits(ops, dtype, rows, vocab, top):
    z, t = logits(rows, vocab, dtype, 3, masked=True)
    check_grad(ops, z, t, check(ops, z, t, top, 1.0), top, 1.0)
    z, t = logits(rows, vocab, dtype, 4, step=2.0)
    check_grad(ops, z, t, check(ops, z, t, top, 1.3), top, 1.3)
    z = torch.full((rows, vocab), 1.5).to(dtype)
    z[:, ::3] = 0.0
    z[:, 1::3] = -0.0
    z[0] = LOWEST[dtype]
    z[1] = 0.0
    z[2, : vocab // 2] = -math.inf
    check(ops, z, t, top, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [40, 700, 6001, 70000])
def test_sorted_rows(ops, dtype, vocab):
    """The largest logits side by side, at the front, at the end, all in one thread's share."""
    base = torch.linspace(-9, 9, vocab)
    steps = [base, base.flip(0), base.roll(vocab // 3)]
    for stride in (8, 32, 256, 2048):
        x = base.clone()
        x[::stride] += 40
        steps.append(x)
    z = torch.stack(steps).to(dtype)
    t = torch.full((len(steps),), vocab - 1)
    r = check(ops, z, t, 20, 1.0)
    check_grad(ops, z, t, r, 20, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [9, 300, 5000, 66001])
def test_rows_without_anything_left(ops, dtype, vocab):
    z, t = logits(4, vocab, dtype, 5)
    z[1] = -math.inf
    z[2] = -math.inf
    z[2, vocab - 2] = 3.0
    z[3, 1:] = LOWEST[dtype]
    t[:] = torch.tensor([0, 3, vocab - 2, 1])
    r = check(ops, z, t, 3, 1.0)
    assert r.top_ids[1].tolist() == [0, 1, 2] and r.lse[1] == -math.inf and r.entropy[1] == 0 and r.logprob[1] == -math.inf
    assert r.entropy[2] == 0 and r.logprob[2] == 0
    g = torch.ones(4, device="cuda")
    d = ops.token_logprobs_grad(z.cuda(), t.cuda(), r, grad_logprob=g, grad_entropy=g, grad_lse=g, grad_top=torch.ones((4, 3), device="cuda"))
    assert not d[1].any() and torch.isfinite(d).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [9, 300, 5000, 66001])
def test_nan_and_infinity(ops, dtype, vocab):
    """A row with NaN or +infinity has no probabilities; its best ids are still the largest numbers', and other rows are as ever."""
    z, t = logits(5, vocab, dtype, 6)
    z[1, 2], z[2, 4], z[3, :], z[4, :] = math.nan, math.inf, math.nan, -math.inf
    z[4, 7] = math.nan
    r = ops.token_logprobs(z.cuda(), t.cuda(), top=4)
    clean = check(ops, z[:1], t[:1], 4, 1.0)
    for a, b in zip(r, clean):
        assert torch.equal(a[:1], b)
    for x in (r.lse[1], r.lse[2], r.lse[3], r.lse[4], r.entropy[1:], r.logprob[1:]):
        assert (x.isnan() | (x == math.inf)).all()
    want = torch.sort(z[1].double().nan_to_num(-math.inf), descending=True, stable=True)[1][:4]
    assert r.top_ids[1].tolist() == want.tolist()
    assert r.top_ids[2, 0] == 4 and r.top_ids[3].tolist() == [0, 1, 2, 3] and r.top_ids[4].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_strides_alignment_and_token_types(ops, dtype):
    for rows, vocab in ((4, 77), (3, 4999), (150, 2000), (2, 30011)):
        z, t = logits(rows, vocab, dtype, 7)
        wide = torch.full((rows, vocab + 13), 50.0, dtype=dtype, device="cuda")
        for shift in (0, 1, 5, 8):
            part = wide[:, shift:shift + vocab]
            part.copy_(z.cuda())
            r = check(ops, z, t.to(torch.int32), 6, 1.0, gpu=part)
            both = torch.stack([t, t + 1], 1).cuda()
            assert all(torch.equal(a, b) for a, b in zip(r, ops.token_logprobs(part, both[:, 0], top=6)))
            check_grad(ops, z, t, r, 6, 1.0, gpu=part, in_place=True)
            edge = torch.cat([wide[:, :shift], wide[:, shift + vocab:]], 1)
            assert (edge == 50).all()
            wide.fill_(50.0)
        one = z[:1].cuda().expand(5, vocab)          # a broadcast row
        r = ops.token_logprobs(one, t[:1].cuda().expand(5), top=2)
        assert all((x == x[0]).all() for x in r)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_through_autograd_and_against_differences(ops, dtype):
    z, t = logits(6, 40, dtype, 8)
    t[2] = -1
    g = torch.Generator().manual_seed(1)
    w = torch.randn((3, 6), generator=g, dtype=torch.float64)
    wt = torch.randn((6, 3), generator=g, dtype=torch.float64)
    ids = ref.logprobs(z, t, 3, 0.8)[3]

    def value(x):
        lp, h, lse, _, _ = ref.logprobs(x, t, 0, 0.8)
        alt = (x.double() / 0.8 - lse[:, None]).gather(1, ids)
        return float((w[0] * lp + w[1] * h + w[2] * lse).sum() + (wt * alt).sum())
    leaf = z.cuda().requires_grad_()
    r = ops.token_logprobs(leaf, t.cuda(), top=3, temperature=0.8)
    loss = (w[0].float().cuda() * r.logprob + w[1].float().cuda() * r.entropy + w[2].float().cuda() * r.lse).sum() + (wt.float().cuda() * r.top_logprobs).sum()
    loss.backward()
    step = 1e-5
    want = torch.zeros_like(z, dtype=torch.float64)
    for i in range(6):
        for j in range(40):
            x = z.double().clone()
            x[i, j] += step
            up = value(x)
            x[i, j] -= 2 * step
            want[i, j] = (up - value(x)) / (2 * step)
    # the differences: third derivatives (below 50) times step^2, and 64-bit rounding of a sum below 200 over the step
    bound = UNIT[dtype] * want.abs() + 50 * step ** 2 + 200 * 2.0 ** -52 / step * 8 + 2.0 ** -18
    assert ((leaf.grad.cpu().double() - want).abs() <= bound).all()
    # sums: a broadcast gradient, of one output alone, and of none of them
    leaf.grad = None
    ops.token_logprobs(leaf, t.cuda()).logprob.sum().backward()
    only, _ = ref.logprobs_grad(z, t, None, torch.ones(6), torch.zeros(6), torch.zeros(6), None, 1.0)
    assert ((leaf.grad.cpu().double() - only).abs() <= UNIT[dtype] * only.abs() + 2.0 ** -18).all()


def test_streams_graphs_and_repeats(ops):
    z, t = logits(33, 40007, BF16, 9, step=0.25)
    z, t = z.cuda(), t.cuda()
    want = ops.token_logprobs(z, t, top=20)
    grad = ops.token_logprobs_grad(z, t, want, grad_logprob=want.logprob, grad_top=want.top_logprobs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = ops.token_logprobs(z, t, top=20)
        cap_grad = ops.token_logprobs_grad(z, t, cap, grad_logprob=cap.logprob, grad_top=cap.top_logprobs)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        for s in side:
            with torch.cuda.stream(s):
                outs.append(ops.token_logprobs(z, t, top=20))
    graph.replay()
    torch.cuda.synchronize()
    for r in outs + [cap]:
        assert all(torch.equal(a, b) for a, b in zip(r, want))
    assert torch.equal(cap_grad, grad)


def test_refusals(ops):
    from paper_2507_23777_b200.binding import XsmError
    z, t = torch.zeros((2, 10), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    r = ops.token_logprobs(z, t, top=2)
    both = (ValueError, XsmError)
    for call in (lambda: ops.token_logprobs(z[0], t), lambda: ops.token_logprobs(z.double(), t), lambda: ops.token_logprobs(z.t(), t), lambda: ops.token_logprobs(z, t[:1]),
                 lambda: ops.token_logprobs(z, t.float()), lambda: ops.token_logprobs(z.cpu(), t), lambda: ops.token_logprobs(z, t.cpu()),
                 lambda: ops.token_logprobs(z, t, top=11), lambda: ops.token_logprobs(z.repeat(1, 9), t, top=33), lambda: ops.token_logprobs(z, t, top=-1),
                 lambda: ops.token_logprobs(z, t, temperature=0.0), lambda: ops.token_logprobs(z, t, temperature=-1.0), lambda: ops.token_logprobs(z, t, temperature=math.nan),
                 lambda: ops.token_logprobs(z, t, temperature=math.inf), lambda: ops.token_logprobs(z[:, :0], t),
                 lambda: ops.token_logprobs_grad(z, t, r, grad_logprob=torch.zeros(3, device="cuda")), lambda: ops.token_logprobs_grad(z, t, r, grad_top=torch.zeros((2, 3), device="cuda")),
                 lambda: ops.token_logprobs_grad(z, t, r, out=z.to(BF16)), lambda: ops.token_logprobs_grad(z, t, r, out=z[:1].expand(2, 10)),
                 lambda: ops.token_logprobs_grad(z, t, ops.token_logprobs(z[:1], t[:1]))):
        with pytest.raises(both):
            call()
    empty = ops.token_logprobs(z[:0], t[:0], top=2)
    assert empty.logprob.shape == (0,) and empty.top_ids.shape == (0, 2)
    assert ops.token_logprobs_grad(z[:0], t[:0], empty, grad_top=empty.top_logprobs).shape == (0, 10)


def test_derivatives_that_no_call_has_are_refused(ops):
    """Forward mode, and second derivatives: an error, not a result without its derivative."""
    import torch.autograd.forward_ad as forward_ad
    z, t = logits(3, 40, F32, 11)
    z, t, g = z.cuda(), t.cuda(), torch.ones(3, device="cuda")
    r = ops.token_logprobs(z, t, top=2)
    leaf, gl = z.clone().requires_grad_(), g.clone().requires_grad_()
    gt = torch.ones((3, 2), device="cuda", requires_grad=True)
    for call in (lambda: ops.token_logprobs_grad(leaf, t, r, grad_logprob=g), lambda: ops.token_logprobs_grad(2 * leaf, t, r, grad_logprob=g),
                 lambda: ops.token_logprobs_grad(z, t, r, grad_logprob=gl), lambda: ops.token_logprobs_grad(z, t, r, grad_entropy=gl),
                 lambda: ops.token_logprobs_grad(z, t, r, grad_lse=gl), lambda: ops.token_logprobs_grad(z, t, r, grad_top=gt),
                 lambda: ops.token_logprobs_grad(z, t, r, grad_logprob=g, out=2 * leaf),
                 lambda: ops.token_logprobs_grad(z, t, ops.token_logprobs(leaf, t), grad_logprob=g)):
        with pytest.raises(ValueError) as e:
            call()
        assert "no_grad" in str(e.value)
        with torch.no_grad():
            call()
    kp = torch.zeros((4, 2, 32, 64), dtype=BF16, device="cuda")
    cache = ops.PagedCache(kp, kp.clone())
    table, one = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    x = torch.zeros((1, 1, 2, 64), dtype=BF16, device="cuda")
    with forward_ad.dual_level():
        dual, dual_x, dual_g = (forward_ad.make_dual(a, torch.ones_like(a)) for a in (z, x, g))
        for call in (lambda: ops.token_logprobs(dual, t), lambda: ops.token_logprobs_grad(dual, t, r, grad_logprob=g), lambda: ops.token_logprobs_grad(z, t, r, grad_logprob=dual_g),
                     lambda: cache.append(dual_x, x, table, one), lambda: cache.append(x, x, table, one, q=dual_x), lambda: cache.attend(dual_x, table, one)):
            with pytest.raises(ValueError) as e:
                call()
            assert "forward" in str(e.value)
        assert all(torch.equal(a, b) for a, b in zip(ops.token_logprobs(z, t, top=2), r))          # what has no tangent is as ever
    with pytest.raises(Exception):
        torch.func.jvp(lambda a: ops.token_logprobs(a, t).logprob, (z,), (z,))


def test_numbers_beyond_their_type_are_refused(ops):
    """(Before any memory is asked for.)"""
    from paper_2507_23777_b200.binding import XsmError
    z, t = torch.zeros((2, 10), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    r = ops.token_logprobs(z, t)
    for call in (lambda: ops.token_logprobs(z, t, top=2 ** 40), lambda: ops.token_logprobs(z, t, top=2 ** 31), lambda: ops.token_logprobs(z, t, top=1.5),
                 lambda: ops.token_logprobs(z, t, temperature=1e39), lambda: ops.token_logprobs_grad(z, t, r, temperature=1e39)):
        with pytest.raises((ValueError, XsmError)):
            call()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("offset", [0.0, 100.0, -100.0, 1000.0, 10000.0, -10000.0])
@pytest.mark.parametrize("rows,vocab", [(9, 50), (5, 3001), (700, 1000), (2, 40001)])
def test_gradient_of_logits_with_an_offset(ops, dtype, offset, rows, vocab):
    """What all logits of a row have in common does not matter, neither for a token that has nearly all of the probability (its gradient is what
    it lacks) nor for one that has little.  Probabilities come from differences to the token's logit, their size times 2^-22; the
    token's own gradient 1 - p is a difference of numbers next to one."""
    z, t = logits(rows, vocab, F32, 12)
    near = torch.arange(rows) % 3
    z[torch.arange(rows), t] = torch.where(near == 0, 24.0, torch.where(near == 1, 12.0, z[torch.arange(rows), t]))
    z = (z + offset).to(dtype)
    g = torch.randn(rows, generator=torch.Generator().manual_seed(2))
    zero = torch.zeros(rows)
    for temperature in (1.0, 0.5):
        gz = z.cuda()
        r = ops.token_logprobs(gz, t.cuda(), temperature=temperature)
        d = ops.token_logprobs_grad(gz, t.cuda(), r, grad_logprob=g.cuda(), temperature=temperature)
        want, size = ref.logprobs_grad(z, t, None, g, zero, zero, None, temperature)
        zd = z.double() / temperature
        depth = (zd - zd.gather(1, t[:, None])).abs() + ref.logprobs(z, t, 0, temperature)[0].abs()[:, None]
        own = torch.zeros_like(want).scatter_(1, t[:, None], g.abs().double()[:, None])
        same(d, want, UNIT[dtype] * want.abs() + (depth * 2.0 ** -22 + (vocab / 256 + 40) * 2.0 ** -24 + 2.0 ** -20) * size + 2.0 ** -21 * own / temperature + TINY[dtype], "gradient")
        leaf = z.cuda().requires_grad_()
        (g.cuda() * ops.token_logprobs(leaf, t.cuda(), temperature=temperature).logprob).sum().backward()
        assert torch.equal(leaf.grad, d)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gradient_where_the_token_is_masked_or_all_logits_are_the_lowest(ops, dtype):
    """Tokens whose own logit says nothing about the others: -infinity, the type's lowest number; rows that hold nothing but that."""
    z, t = logits(6, 300, dtype, 13)
    z[0, t[0]], z[1, t[1]], z[2] = -math.inf, LOWEST[dtype], LOWEST[dtype]
    t[3] = -1
    r = ops.token_logprobs(z.cuda(), t.cuda(), top=4)
    check_grad(ops, z, t, r, 4, 1.0)
    r = ops.token_logprobs(z.cuda(), t.cuda(), top=4, temperature=0.5)
    d = ops.token_logprobs_grad(z.cuda(), t.cuda(), r, grad_logprob=torch.ones(6, device="cuda"), temperature=0.5)
    want = torch.full((300,), -2.0 / 300, dtype=torch.float64)
    want[t[2]] += 2
    same(d[2], want, UNIT[dtype] * want.abs() + 2.0 ** -20, "all the lowest")
