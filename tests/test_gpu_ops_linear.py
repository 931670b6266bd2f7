"""Log probabilities from hidden states without the logits, and their gradients, against plain torch in 64 bits."""
import math

import pytest
import torch

import block_reference as ref
from block_reference import BF16, F16, F32, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "this test needs a B200"
    from paper_2507_23777_b200 import build, ops
    build.build()
    yield ops
    ops.check()


def inputs(rows, vocab, d, dtype, seed=0, spread=2.0, padding=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((rows, d), generator=g, device="cuda").to(dtype)
    w = (spread * d ** -0.5 * torch.randn((vocab, d), generator=g, device="cuda")).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    if padding:
        t[padding - 1::padding] = -1
    gl, gs = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    return h, w, t, gl, gs


def check(ops, h, w, t, gl, gs, temperature=1.0, forward_only=False):
    r = ops.linear_logprobs(h, w, t, temperature)
    few = h.shape[0] <= 128 or w.shape[0] <= 64        # (a CTA a tile)
    logprob, lse, _, b_logprob, b_lse, _ = ref.linear(h, w, t, temperature, few)
    near(r.lse, lse, b_lse, "lse")
    near(r.logprob, logprob, b_logprob, "logprob")
    if not forward_only:
        got = ops.linear_logprobs_grad(h, w, t, r, gl, gs, temperature)
        for x, (want, bound), what in zip(got, ref.linear_grad(h, w, t, temperature, gl, gs, 2 if few else 1), ("d_hidden", "d_weight")):
            assert x.dtype is h.dtype and x.is_contiguous()
            near(x, want, bound, what)
    return r


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 8), (1, 50, 64), (5, 64, 72), (7, 65, 24), (8, 4096, 256), (16, 1000, 768), (33, 257, 512), (96, 20011, 128), (127, 300, 200), (128, 129, 64),
                                          (129, 256, 64), (129, 65, 72), (200, 64, 1024), (256, 257, 96), (300, 5003, 768), (513, 511, 320), (1000, 2000, 1024), (2049, 100, 136), (2, 300, 4104), (90, 400, 4096), (7, 130, 1032), (128, 70, 1272), (31, 5000, 2040)])
def test_sizes(ops, dtype, rows, vocab, d):
    check(ops, *inputs(rows, vocab, d, dtype, seed=rows + vocab + d))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,d", [(3, 700, 256), (300, 700, 256)])
@pytest.mark.parametrize("temperature", [0.05, 0.7, 30.0])
def test_temperatures(ops, dtype, rows, vocab, d, temperature):
    check(ops, *inputs(rows, vocab, d, dtype, seed=1), temperature=temperature)


@pytest.mark.parametrize("rows,d", [(70001, 64), (70001, 72), (150001, 136)])
def test_vocabulary_in_pieces(ops, rows, d):
    """More rows times tokens than one piece of the gradients by the logits takes: sums over the pieces are added up in fp32."""
    h, w, t, gl, gs = inputs(rows, 2500, d, BF16, seed=2)
    r = ops.linear_logprobs(h, w, t)
    d_hidden, d_weight = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    some = torch.cat([torch.arange(300, device="cuda"), torch.arange(rows - 300, rows, device="cuda")])
    (want, bound), _ = ref.linear_grad(h[some], w, t[some], 1.0, gl[some], gs[some])
    near(d_hidden[some], want, bound + want.abs() * 2.0 ** -22, "d_hidden")
    want, bound = 0.0, 0.0
    for a in range(0, rows, 30000):
        _, (x, b) = ref.linear_grad(h[a:a + 30000], w, t[a:a + 30000], 1.0, gl[a:a + 30000], gs[a:a + 30000])
        want, bound = want + x, bound + b
    near(d_weight, want, bound * (rows / 30000 + 1), "d_weight")        # (the accumulator holds all rows' sum while it takes the last of them)


@pytest.mark.parametrize("size", [1.0, 2.0 ** -30])
def test_many_rows_in_fp16(ops, size):
    """More rows than every CTA looks through for the largest gradient, and a vocabulary in pieces (gradients of one size: the scale is then every row's)."""
    rows = 70001
    h, w, t, gl, gs = inputs(rows, 2500, 64, F16, seed=20)
    w = w * 8
    gl, gs = 2 * size * gl.sign(), size * gs.sign()
    r = ops.linear_logprobs(h, w, t)
    d_hidden, d_weight = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    some = torch.cat([torch.arange(300, device="cuda"), torch.arange(rows - 300, rows, device="cuda")])
    t[:5] = 3
    (want, bound), _ = ref.linear_grad(h[some[5:]], w, t[some[5:]], 1.0, gl[some[5:]], gs[some[5:]])
    near(d_hidden[some[5:]], want, bound + want.abs() * 2.0 ** -22, "d_hidden")
    alone = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(False, True))
    assert alone[0] is None and alone[1].isfinite().all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,vocab,d", [(9000, 40, 72), (9001, 150, 128), (20, 30011, 64), (300, 60001, 256), (20001, 8, 8)])
def test_long_sums_of_few_tiles(ops, dtype, rows, vocab, d):
    """Sums that are cut into many, of either gradient."""
    check(ops, *inputs(rows, vocab, d, dtype, seed=21))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [4, 260])
def test_only_some_gradients(ops, dtype, rows):
    h, w, t, gl, gs = inputs(rows, 900, 128, dtype, seed=3)
    r = ops.linear_logprobs(h, w, t)
    both = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    a = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(True, False))
    b = ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(False, True))
    assert a[1] is None and b[0] is None and torch.equal(a[0], both[0]) and torch.equal(b[1], both[1])
    assert ops.linear_logprobs_grad(h, w, t, r, gl, gs, need=(False, False)) == (None, None)
    for g, s in ((gl, None), (None, gs), (None, None)):
        for x, (want, bound) in zip(ops.linear_logprobs_grad(h, w, t, r, g, s), ref.linear_grad(h, w, t, 1.0, g, s)):
            near(x, want, bound, "gradient")


@pytest.mark.parametrize("size", [2.0 ** -30, 1e-6, 1e4, 2.0 ** 40])
def test_gradients_of_any_size_in_fp16(ops, size):
    """The gradients by the logits are scaled to the type's range; what leaves the type's range in the result is zero or infinite as a rounding is."""
    h, w, t, gl, gs = inputs(300, 400, 64, F16, seed=4)
    r = ops.linear_logprobs(h, w, t)
    gl, gs = gl * size, gs * size
    for x, (want, bound) in zip(ops.linear_logprobs_grad(h, w, t, r, gl, gs), ref.linear_grad(h, w, t, 1.0, gl, gs)):
        sure = (want.abs() + bound < 65000) | (want.abs() - bound > 66000)
        near(torch.where(sure, x.double(), 0.0), torch.where(sure, torch.where(want.abs() > 65519, want.sign() * math.inf, want), 0.0), bound, "gradient")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [6, 300])
def test_tokens_outside_the_vocabulary_are_none(ops, dtype, rows):
    h, w, t, gl, gs = inputs(rows, 500, 64, dtype, seed=5, padding=0)
    t[:6] = torch.tensor([-1, 500, 2 ** 31, -2 ** 40, 2 ** 62, -2 ** 63], device="cuda")
    r = check(ops, h, w, t, gl, gs)
    assert (r.logprob[:6] == 0).all()
    d = ops.linear_logprobs_grad(h, w, t, r, gl)
    assert (d[0][:6] == 0).all()


@pytest.mark.parametrize("rows", [6, 300])
def test_token_types_strides_and_slices(ops, rows):
    h, w, t, gl, gs = inputs(rows, 700, 128, BF16, seed=6)
    want = ops.linear_logprobs(h, w, t)
    grads = ops.linear_logprobs_grad(h, w, t, want, gl, gs)
    big = torch.full((rows, 3 * 128), math.nan, device="cuda", dtype=BF16)
    big[:, 128:256] = h
    bw = torch.full((900, 256), math.nan, device="cuda", dtype=BF16)
    bw[100:800, :128] = w
    t2 = torch.stack([t.int(), torch.full_like(t.int(), 7)], 1)
    g2 = torch.stack([gl, gs], 1)
    got = ops.linear_logprobs(big[:, 128:256], bw[100:800, :128], t2[:, 0])
    assert torch.equal(got.lse, want.lse) and torch.equal(got.logprob, want.logprob)
    for x, y in zip(ops.linear_logprobs_grad(big[:, 128:256], bw[100:800, :128], t2[:, 0], got, g2[:, 0], g2[:, 1]), grads):
        assert torch.equal(x, y)
    one = torch.full((1,), 0.5, device="cuda").expand(rows)          # as a mean's gradient comes
    for x, y in zip(ops.linear_logprobs_grad(h, w, t, want, one), ops.linear_logprobs_grad(h, w, t, want, one.contiguous())):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [5, 280])
def test_infinities_and_nan_stay_in_their_rows(ops, dtype, rows):
    h, w, t, gl, gs = inputs(rows, 300, 64, dtype, seed=7, padding=0)
    w[:, 0] = -w[:, 0].abs() - 0.25
    clean = ops.linear_logprobs(h, w, t)
    d_clean = ops.linear_logprobs_grad(h, w, t, clean, gl, gs, need=(True, False))[0]
    h2 = h.clone()
    h2[0, 3], h2[1, 0], h2[2, 0] = math.nan, math.inf, -math.inf         # NaN; every logit -inf; every logit +inf
    r = ops.linear_logprobs(h2, w, t)
    d = ops.linear_logprobs_grad(h2, w, t, r, gl, gs, need=(True, False))[0]
    assert r.lse[0].isnan() and r.logprob[0].isnan() and d[0].isnan().all()
    assert r.lse[1] == -math.inf and r.logprob[1] == -math.inf and (d[1] == 0).all()
    assert r.lse[2].isnan() and r.logprob[2].isnan() and d[2].isnan().all()
    assert torch.equal(r.lse[3:], clean.lse[3:]) and torch.equal(r.logprob[3:], clean.logprob[3:]) and torch.equal(d[3:], d_clean[3:])
    # a token of which nothing is left: probability zero
    w2 = w.clone()
    w2[17, 1], h3 = -math.inf, h.abs() + 0.25
    t[:] = 17
    r = ops.linear_logprobs(h3, w2, t)
    assert (r.logprob == -math.inf).all() and r.lse.isfinite().all()
    keep = torch.arange(300, device="cuda") != 17
    near(r.lse, torch.logsumexp((h3.double() @ w.double().T)[:, keep], -1), ref.linear(h3, w, t, 1.0)[4], "lse")


def test_empty_calls(ops):
    h, w, t, gl, gs = inputs(4, 100, 64, BF16)
    r = ops.linear_logprobs(h[:0], w, t[:0])
    assert r.lse.shape == r.logprob.shape == (0,)
    d_hidden, d_weight = ops.linear_logprobs_grad(h[:0], w, t[:0], r, gl[:0])
    assert d_hidden.shape == (0, 64) and d_weight.shape == (100, 64) and (d_weight == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [6, 300])
def test_autograd_and_differences(ops, dtype, rows):
    """Through autograd as by the explicit call; and the slope along a direction against differences of the forward kernel: steps that the type holds, the
    differences' own error taken from 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(8)
    h = (torch.randint(-12, 13, (rows, 64), generator=g, device="cuda") / 8).to(dtype).requires_grad_()
    w = (torch.randint(-12, 13, (200, 64), generator=g, device="cuda") / 32).to(dtype).requires_grad_()
    t = torch.randint(-1, 200, (rows,), generator=g, device="cuda")
    gl, gs = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    r = ops.linear_logprobs(h, w, t, temperature=1.3)
    d_h, d_w = torch.autograd.grad((r.logprob * gl).sum() + (r.lse * gs).sum(), [h, w])
    with torch.no_grad():
        for x, y in zip(ops.linear_logprobs_grad(h, w, t, r, gl, gs, 1.3), (d_h, d_w)):
            assert torch.equal(x, y)
        (eh, bh), (ew, bw) = ref.linear_grad(h, w, t, 1.3, gl, gs)
        vh, vw = torch.randint(-1, 2, h.shape, generator=g, device="cuda").double(), torch.randint(-1, 2, w.shape, generator=g, device="cuda").double()
        for which, step in ((0, 0.125), (1, 0.03125)):
            def at(s):
                a, b = (h + s * step * vh, w) if which == 0 else (h, w + s * step * vw)
                a, b = a.to(dtype), b.to(dtype)
                k = ops.linear_logprobs(a, b, t, temperature=1.3)
                e = ref.linear(a, b, t, 1.3)
                return ((k.logprob.double() * gl).sum() + (k.lse.double() * gs).sum(), (e[0] * gl).sum() + (e[1] * gs).sum(), (e[3] * gl.abs()).sum() + (e[4] * gs.abs()).sum())
            plus, minus = at(1), at(-1)
            slope, exact = (plus[0] - minus[0]) / (2 * step), (plus[1] - minus[1]) / (2 * step)
            v, e, b, got = (vh, eh, bh, d_h) if which == 0 else (vw, ew, bw, d_w)
            own = (exact - (e * v).sum()).abs()          # what the differences themselves are off
            assert abs(slope - (got.double() * v).sum()) <= own + (plus[2] + minus[2]) / (2 * step) + (b * v.abs()).sum()
            assert own < 0.3 * (e * v).sum().abs() + 1.0        # (they say something)
    for need in ((h, w.detach()), (h.detach(), w)):
        r = ops.linear_logprobs(*need, t, temperature=1.3)
        leaf = h if need[0] is h else w
        assert torch.equal(torch.autograd.grad((r.logprob * gl).sum() + (r.lse * gs).sum(), leaf)[0], d_h if leaf is h else d_w)
    (d,) = torch.autograd.grad(ops.linear_logprobs(h, w, t).logprob.mean(), h)
    with torch.no_grad():
        r = ops.linear_logprobs(h, w, t)
        assert torch.equal(d, ops.linear_logprobs_grad(h, w, t, r, torch.full((rows,), 1.0 / rows, device="cuda"), need=(True, False))[0])


@pytest.mark.parametrize("rows,vocab", [(5, 3000), (300, 3000)])
def test_streams_graphs_and_repeats(ops, rows, vocab):
    h, w, t, gl, gs = inputs(rows, vocab, 256, F16, seed=9)
    r = ops.linear_logprobs(h, w, t)
    d = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    other = inputs(rows, vocab, 256, F16, seed=10)
    r2 = ops.linear_logprobs(*other[:3])
    d2 = ops.linear_logprobs_grad(*other[:3], r2, *other[3:])
    static = [x.clone() for x in (h, w, t, gl, gs)]
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cr = ops.linear_logprobs(*static[:3])
            cd = ops.linear_logprobs_grad(*static[:3], cr, *static[3:])
        graphs.append((graph, cr, cd))
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(8):
        for s in sides:
            with torch.cuda.stream(s):
                x = ops.linear_logprobs(h, w, t)
                outs.append((x, ops.linear_logprobs_grad(h, w, t, x, gl, gs)))
    graphs[0][0].replay()
    torch.cuda.synchronize()
    for x, y in outs + [graphs[0][1:]]:
        assert torch.equal(x.lse, r.lse) and torch.equal(x.logprob, r.logprob) and torch.equal(y[0], d[0]) and torch.equal(y[1], d[1])
    for x, y in zip(static, other):
        x.copy_(y)
    with torch.cuda.stream(sides[0]):
        graphs[1][0].replay()
    with torch.cuda.stream(sides[1]):
        graphs[0][0].replay()
    torch.cuda.synchronize()
    for _, x, y in graphs:
        assert torch.equal(x.lse, r2.lse) and torch.equal(x.logprob, r2.logprob) and torch.equal(y[0], d2[0]) and torch.equal(y[1], d2[1])


def test_a_backward_pass_is_recorded_beside_an_eager_one_of_its_stream(ops):
    """Leaves belong to the stream on which a graph of theirs was made first: torch records their backward pass on that stream."""
    h, w, t, gl, gs = inputs(300, 500, 64, BF16, seed=11)
    h.requires_grad_()
    w.requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = ops.linear_logprobs(h, w, t).logprob          # lives while the other is recorded
        want = torch.autograd.grad((ops.linear_logprobs(h, w, t).logprob * gl).sum(), [h, w])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = torch.autograd.grad((ops.linear_logprobs(h, w, t).logprob * gl).sum(), [h, w])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    with torch.cuda.stream(side):
        again = torch.autograd.grad((eager * gl).sum(), [h, w])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(again, want))


def test_offsets_beyond_32_bits(ops):
    """A vocabulary's weights of 2^31 elements and more."""
    d, vocab = 8192, 270_001
    g = torch.Generator(device="cuda").manual_seed(12)
    w = torch.empty((vocab, d), dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=g)
    for rows in (3, 130):
        h = torch.randn((rows, d), generator=g, device="cuda").to(BF16)
        t = torch.randint(vocab - 5, vocab, (rows,), generator=g, device="cuda")
        r = ops.linear_logprobs(h, w, t)
        z = torch.cat([h[:3].double() @ w[a:a + 20000].double().T for a in range(0, vocab, 20000)], 1)
        want = torch.logsumexp(z, -1)
        bound = (d / 16 + 2) * 2.0 ** -23 * float((h[:3].double().abs() @ w[-2000:].double().abs().T).max()) * 1.2 + float(z.abs().max()) * 2.0 ** -21 + (vocab / 64 + 40) * 2.0 ** -24 + 2.0 ** -20
        near(r.lse[:3], want, torch.full_like(want, bound), "lse")
        near(r.logprob[:3], z.gather(1, t[:3, None])[:, 0] - want, torch.full_like(want, 2 * bound), "logprob")


@pytest.mark.parametrize("rows", [3, 130])
def test_gradients_beyond_32_bits(ops, rows):
    """The last rows of a weight gradient of 2^31 elements and more, and the gradient by hidden, to which they add."""
    d, vocab, last = 8192, 270_001, 40
    g = torch.Generator(device="cuda").manual_seed(22)
    w = torch.empty((vocab, d), dtype=BF16, device="cuda").normal_(0.0, 0.02, generator=g)
    h = torch.randn((rows, d), generator=g, device="cuda").to(BF16)
    t = torch.randint(vocab - last, vocab, (rows,), generator=g, device="cuda")
    gl, gs = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    r = ops.linear_logprobs(h, w, t)
    d_hidden, d_weight = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    tail = w[-last:].double()
    dz = -torch.exp(h.double() @ tail.T - r.lse.double()[:, None]) * (gl - gs).double()[:, None]
    dz[torch.arange(rows, device="cuda"), t - (vocab - last)] += gl.double()
    want = dz.T @ h.double()
    size = dz.abs().T @ h.double().abs()
    # the middle part's rounding, the exponent's error (512 sums cut off, sizes to 20), the result's rounding
    near(d_weight[-last:], want, size * (2.0 ** -8 + 2.0 ** -9) + want.abs() * 2.0 ** -8 + 1e-30, "d_weight")
    dh = torch.zeros((3, d), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(dh)
    for a in range(0, vocab, 20000):
        x = w[a:a + 20000].double()
        p = -torch.exp(h[:3].double() @ x.T - r.lse[:3].double()[:, None]) * (gl - gs)[:3].double()[:, None]
        at = t[:3] - a
        here = (at >= 0) & (at < x.shape[0])
        p[here.nonzero()[:, 0], at[here]] += gl[:3][here].double()
        dh += p @ x
        size += p.abs() @ x.abs()
    near(d_hidden[:3], dh, size * (2.0 ** -8 + 2.0 ** -9) + dh.abs() * 2.0 ** -8, "d_hidden")


@pytest.mark.parametrize("rows", [5, 300])
def test_a_wait_that_runs_out_is_told(ops, rows):
    h, w, t, gl, gs = inputs(rows, 500, 256, BF16, seed=13)
    r = ops.linear_logprobs(h, w, t)
    d = ops.linear_logprobs_grad(h, w, t, r, gl, gs)
    from paper_2507_23777_b200 import binding
    lib = binding.load()
    try:
        lib.xsm_debug_product_waits(2000, 1)
        ops.linear_logprobs(h, w, t)
        with pytest.raises(binding.XsmError, match="patience"):
            ops.check()
        ops.linear_logprobs_grad(h, w, t, r, gl, gs)
        with pytest.raises(binding.XsmError, match="patience"):
            ops.check()
    finally:
        lib.xsm_debug_product_waits(0, 0)
    ops.check()
    again = ops.linear_logprobs(h, w, t)
    assert torch.equal(again.lse, r.lse)
    assert all(torch.equal(x, y) for x, y in zip(ops.linear_logprobs_grad(h, w, t, again, gl, gs), d))
    ops.check()


def test_refusals(ops):
    h, w, t, gl, gs = inputs(4, 100, 64, BF16)
    r = ops.linear_logprobs(h, w, t)
    for bad in (dict(hidden=h.float(), weight=w.float()), dict(weight=w.half()), dict(hidden=h[:, :60], weight=w[:, :60]), dict(weight=w[:, :56]), dict(hidden=h[0]), dict(hidden=h.T),
                dict(weight=w[:0]), dict(tokens=t[:3]), dict(tokens=t.float()), dict(tokens=t.cpu()), dict(hidden=h.cpu()), dict(weight=w.cpu()), dict(temperature=0.0),
                dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=1e-45), dict(hidden=h[:1].expand(4, -1)),
                dict(hidden=torch.zeros(4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(4, 64)), dict(hidden=torch.zeros((4, 68), dtype=BF16, device="cuda")[:, :64])):
        args = dict(hidden=h, weight=w, tokens=t)
        args.update(bad)
        with pytest.raises((ValueError, RuntimeError)):
            ops.linear_logprobs(**args)
        with pytest.raises((ValueError, RuntimeError)):
            ops.linear_logprobs_grad(**args, result=r, grad_logprob=gl)
    for bad in (dict(grad_logprob=gl[:3]), dict(grad_logprob=gl.double()), dict(grad_lse=gl.cpu()), dict(result=(None, r.lse[:3])), dict(result=(None, r.lse.double()))):
        args = dict(result=r, grad_logprob=gl)
        args.update(bad)
        with pytest.raises(ValueError):
            ops.linear_logprobs_grad(h, w, t, **args)
    hg = h.clone().requires_grad_()
    with pytest.raises(ValueError, match="no_grad"):
        ops.linear_logprobs_grad(hg, w, t, r, gl)
    x = ops.linear_logprobs(hg, w, t)
    (g1,) = torch.autograd.grad(x.logprob.sum(), hg, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g1.float().sum(), hg)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            ops.linear_logprobs(torch.autograd.forward_ad.make_dual(h, h.clone()), w, t)
